"""Calls on one pool in 8 bits at the same time on several streams; the summaries and the decode over a prefix that was served in 8 bits; pieces of the chunk kernel
that outlast its page table."""
import dataclasses

import numpy as np
import pytest
import torch

import paged_utils as P
import quant_utils as Q
from paper_2604_05438_amd import binding as B
from paper_2604_05438_amd import inputs as I
from paper_2604_05438_amd.paged import PagedCache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,lens", [(16, (40000, 20)), (1, (5000, 20)), (7, (20000, 9))])
@pytest.mark.parametrize("window", [0, 4500])
def test_long_pieces_of_64_channels_in_the_chunk_kernel(page, lens, window):
    """One workgroup passes over more pages than it holds the page table of; 7 query heads per KV head, so that the rows are more than the split kernel takes"""
    st = Q.Step(14, 2, 64, [lens, (3, 1)], page, seed=4).upload()
    assert st.max_new * 7 > 32
    out, lse = st.call(B.tkphi_quant_attention, st.config(window=window, workgroups=1))
    P.check(st, out, lse, P.attention_oracle(st, window=window))


def test_attention_and_an_append_to_one_pool_at_once():
    """Sequences of one pool by twos: single tokens over what is cached, a chunk over what is cached, an append; each call on a stream and a workspace of its own.  As one
    after another, to the bit; the attention also against the oracle."""
    hq, hkv, d = 14, 2, 64
    st = Q.Step(hq, hkv, d, [(3000, 1), (700, 2), (900, 40), (10, 33), (60, 500), (7, 100)], 32, block=16, seed=1).upload()
    t = st.dev
    gen = torch.Generator(device="cuda").manual_seed(3)
    new = [m for _, m in st.lens]
    rows = torch.randn(600, hq + 2 * hkv, d, generator=gen, device="cuda").bfloat16()
    q_rot = torch.empty(600, hq, d, device="cuda", dtype=torch.bfloat16)
    freq = torch.from_numpy(500000.0 ** (-np.arange(0, d, 2) / d)).cuda()
    seqs = t["seqs"].clone()
    seqs[4:, 2] -= st.first[4]                               # (the append has rows of its own)
    cfg, pool = st.config(rot_dim=d), st.pool()
    parts = []
    for i, n_rows in ((0, st.rows), (2, st.rows), (4, 600)):
        step = B.make_step(seqs[i:i + 2], t["pages"][i:i + 2], n_rows, max(new[i:i + 2]), st.max_len)
        parts.append((step, B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step)), torch.cuda.Stream()))
    att = B.make_attention_rows(t["q"], t["out"], t["lse"])
    app = B.make_new_rows(rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:], q_rot, inv_freq=freq)
    changed = [t["K8"].view(torch.uint8), t["V8"].view(torch.uint8), t["S"], t["M"], q_rot, t["out"], t["lse"]]
    before = [x.clone() for x in changed]

    def calls(streams):
        for k, (step, ws, stream) in enumerate(parts):
            with torch.cuda.stream(stream if streams else torch.cuda.current_stream()):
                tail = (ws.data_ptr(), ws.numel(), B.current_stream_ptr())
                if k < 2:
                    B.tkphi_quant_attention(cfg, step, pool, att, *tail)
                else:
                    B.tkphi_quant_append(cfg, step, pool, app, None, *tail)

    calls(False)
    torch.cuda.synchronize()
    want = [x.clone() for x in changed]
    assert not torch.equal(want[0], before[0]) and not torch.equal(want[3], before[3])
    for _ in range(5):
        for x, y in zip(changed, before):
            x.copy_(y)
        torch.cuda.synchronize()
        for _ in range(8):
            calls(True)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(changed, want))
    for _, ws, _ in parts:
        assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == 0
    P.check(st, t["out"].double().cpu().numpy(), t["lse"].double().cpu().numpy(), P.attention_oracle(st), skip=(4, 5))


@pytest.mark.parametrize("shape,L,k,heads_first", [("l1b_32k", 2500, 24, True), ("l3b_128k", 3001, 29, False)])
def test_summaries_and_decode_over_a_prefix_read_back(shape, L, k, heads_first):
    """A prompt appended in chunks to a cache of codes, read back in several calls as [KV heads][rows][channels]; the summary build and the decode over those rows against the
    oracle over the same rows"""
    import parity_utils as PU
    from paper_2604_05438_amd import harness as H
    w = dataclasses.replace(I.WORKLOADS[shape], n_needles=0)
    hkv, d = w.n_kv_heads, w.d_head
    layer = I.make_layer(w, L=L)
    k_rows, v_rows = (H.to_device(layer[n]).transpose(0, 1) for n in "KV")
    c = PagedCache(w.n_q_heads, hkv, d, -(-L // 64) + 2, 64, 1, 1000, L, heads_first=heads_first, codes=True)
    for a in range(0, L, 1000):
        n = min(1000, L - a)
        c.begin_step({"prompt": n})
        c.append(None, k_rows[a:a + n], v_rows[a:a + n], None)
        c.end_step()
    K, V = torch.full((2, hkv, L + 5, d), 7.0, device="cuda", dtype=torch.bfloat16)
    c.read("prompt", K.transpose(0, 1), V.transpose(0, 1))
    assert c.status() == 0 and (K[:, L:] == 7).all() and (V[:, L:] == 7).all()
    assert ((V[:, :L] - v_rows.transpose(0, 1)).float().abs() <= 2.0 ** -4 * v_rows.transpose(0, 1).float().abs() + 2.0 ** -14).all()
    b = H.Batch(H.config_of(w), [dict(layer, K=K, V=V)], [k], debug=True)
    b.build()
    b.decode()
    assert b.status() == 0
    host = {n: x.view(torch.int16).cpu().numpy().view(np.uint16) for n, x in (("K", K), ("V", V))}
    PU.check_layer(w, dict(layer, **host), k, b, 0)
