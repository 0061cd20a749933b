"""The serving example with normed heads and on a cache in 8 bits, every output against the oracle; a prefix read back, and what is built on it."""
import os
import sys

import numpy as np
import pytest
import torch

from paper_2604_05438_amd import binding as B
from paper_2604_05438_amd.paged import PagedCache

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,codes,normed", [("bf16", False, True), ("f32", False, True), ("bf16", True, False), ("bf16", True, True)])
def test_serving_loop(dtype, codes, normed):
    import paged_serving
    assert paged_serving.check(dtype, codes, normed) <= 1.0


def test_prefix_read_back_in_the_layout_of_contiguous_caches():
    """Two prompts appended in chunks; one read back, in more calls than one, as [KV heads][rows][channels]"""
    gen = torch.Generator(device="cuda").manual_seed(4)
    c = PagedCache(8, 2, 64, 40, 16, 2, 100, 400, block=16, first_blocks=1, last_blocks=1, top_blocks=4, codes=True)
    kept = {"a": [], "b": []}
    for new in ({"a": 60, "b": 40}, {"b": 33, "a": 1}, {"a": 90}, {"a": 100}):
        c.begin_step(new)
        rows = sum(new.values())
        qkv = torch.randn(rows, 12, 64, generator=gen, device="cuda").bfloat16()
        q_rot = torch.empty(rows, 8, 64, device="cuda", dtype=torch.bfloat16)
        c.append(qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], q_rot)
        at = 0
        for s, m in new.items():
            kept[s].append(qkv[at:at + m, 10:])
            at += m
        c.end_step()
    K, V = torch.full((2, 2, 260, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    c.read("a", K.transpose(0, 1), V.transpose(0, 1))
    assert c.status() == 0
    v = torch.cat(kept["a"]).transpose(0, 1).float()
    top = v.abs().amax(-1, keepdim=True)
    # half a step of the code, or of the least one (2^-10 of the power of two, which is below 2^-7 of the row's largest element)
    assert ((V[:, :251].float() - v).abs() <= torch.maximum(2.0 ** -4 * v.abs(), 2.0 ** -17 * top)).all()
    assert (V[:, 251:] == 7).all() and (K[:, 251:] == 7).all()
    pages = torch.tensor(c.pages["a"], device="cuda")
    t = torch.arange(251, device="cuda")
    scale = torch.exp2(c.scales.float() - 127)
    want = (c.K.float() * scale[..., :1])[pages[t // 16], :, t % 16].transpose(0, 1)
    assert torch.equal(K[:, :251].float(), want)
    c.read("b", None, V.transpose(0, 1))
    assert (V[:, 73:251] != 7).any()


def test_two_workspaces_on_two_streams_at_once():
    """Attention over codes, and an append to other pages, at the same time, each with a workspace of its own"""
    import paged_utils as P
    import quant_utils as Q
    one, two = Q.Step(14, 2, 64, [(3000, 1), (700, 2)], 32, seed=1).upload(), Q.Step(10, 2, 128, [(500, 40)], 16, seed=2).upload()
    streams = [torch.cuda.Stream() for _ in range(2)]
    want = [s.call(B.tkphi_quant_attention, s.config())[0] for s in (one, two)]
    sizes = [B.tkphi_paged_workspace_bytes(s.config(), s.step()) for s in (one, two)]
    spaces = [B.alloc_paged_workspace(n) for n in sizes]
    for s in (one, two):
        s.dev["out"].fill_(7.0)
    torch.cuda.synchronize()
    keep = []
    for _ in range(20):
        for s, stream, ws in zip((one, two), streams, spaces):
            with torch.cuda.stream(stream):
                keep.append((s.step(), B.make_attention_rows(s.dev["q"], s.dev["out"], s.dev["lse"])))
                B.tkphi_quant_attention(s.config(), keep[-1][0], s.pool(), keep[-1][1], ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    torch.cuda.synchronize()
    for s, w in zip((one, two), want):
        assert np.array_equal(s.dev["out"].double().cpu().numpy(), w)
    P.check(one, one.dev["out"].double().cpu().numpy(), None, P.attention_oracle(one))
