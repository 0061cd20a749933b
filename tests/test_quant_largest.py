"""The largest finite numbers in a cache in 8 bits: an element that is finite is stored as a finite number, within 2^-4 of it."""
import numpy as np
import pytest
import torch

import quant_utils as Q
from oracle import paged_oracle as O
from paper_2604_05438_amd import binding as B

LARGEST = [n * 2.0 ** 120 for n in (255, 254, 249, 248, 247, 241, 240, 239, 232, 224, 223, 128)]       # every code next to 256 x 2^120 = 2^128 among them


def rows(count, d):
    """Rows [count][d] of bf16 numbers up to LARGEST, of both signs, down to a tenth"""
    gen = torch.Generator().manual_seed(6)
    x = (torch.rand(count, d, generator=gen) * 2 - 1) * 2.0 ** 127 * 1.5
    for i in range(count):
        x[i, ::5] = LARGEST[i % len(LARGEST)] * (1 if i & 1 else -1)
        x[i, 7] = -x[i, 5]
    return x.bfloat16()


def stored(codes, scales):
    """What the codes stand for, as bf16"""
    return (codes.double() * torch.exp2(scales.double() - 127)[..., None]).bfloat16()


def check(x, values):
    x, y = x.double(), values.double()
    assert torch.isfinite(y).all() and ((y - x).abs() <= 2.0 ** -4 * x.abs() + 2.0 ** 110).all()       # (2^-10 of a power of two, 2^120 at most)


def test_oracle_keeps_them_finite():
    x = rows(24, 64)
    codes, b = O.quantise(x.double().numpy())
    check(x, stored(torch.from_numpy(codes), torch.from_numpy(b)))
    assert b.max() == 247 and np.abs(codes[b == 247]).max() == 240
    codes, b = O.quantise(np.array([[255 * 2.0 ** 120, np.inf, -np.inf, np.nan, -248 * 2.0 ** 120, 247 * 2.0 ** 120]]))
    assert codes[0, [0, 4, 5]].tolist() == [240, -240, 240] and np.isnan(codes[0, 1:4]).all() and b[0] == 247
    assert abs(256 * (1 - 2.0 ** -24) - 240) <= 2.0 ** -4 * 256 * (1 - 2.0 ** -24)                      # the largest number of 32 bits


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", ["as they are", "turned", "normed"])
def test_largest_numbers_are_stored_as_finite_ones(d, form):
    """Keys go to codes from 32 bits, values from bf16.  turned: through a small angle; normed: heads of equal sizes with a weight that makes them the largest numbers"""
    n = 36
    st = Q.Step(2, 2, d, [(0, n)], 16, block=16, seed=3).upload()
    kv = torch.stack([rows(2 * n, d)] * 2, 0).view(2, n, 2, d)
    freq, norms, weight = None, None, None
    if form == "turned":
        kv[0] = (kv[0].float() * 0.73).bfloat16()             # (turned by up to 35 x 2^-6, where sin + cos = 1.374, the largest come close to 2^128)
        kv[0, :, :, d // 2:] = kv[0, :, :, :d // 2]
        freq = torch.full((d // 2,), 2.0 ** -6, dtype=torch.float64, device="cuda")
    if form == "normed":
        kv[0] = torch.sign(kv[0].float()).bfloat16()
        weight = torch.tensor([LARGEST[c % 5] for c in range(d)]).bfloat16().cuda()
        norms = B.make_head_norms(None, weight, 1e-6)
    k, v = kv[0].cuda(), kv[1].cuda()
    cfg, step, t = st.config(rot_dim=d if freq is not None else 0), st.step(), st.dev
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    io = B.make_new_rows(None, k, v, None, inv_freq=freq)
    B.tkphi_quant_append(cfg, step, st.pool(), io, norms, ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    back = torch.empty(2, n, 2, d, device="cuda", dtype=torch.bfloat16)
    B.tkphi_quant_read(cfg, step, st.pool(), B.make_read_rows(back[0], back[1]), ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == 0
    back = back.cpu()
    codes, b = O.quantise(kv[1].double().numpy())            # (values: to the bit)
    assert torch.equal(back[1], stored(torch.from_numpy(codes), torch.from_numpy(b)))
    check(kv[1], back[1])
    want = kv[0].double().numpy()
    if form == "turned":
        want = np.stack([O.rotate(want[i], i, freq.cpu().numpy(), False) for i in range(n)])
    if form == "normed":
        want = O.head_norm(want, weight.double().cpu().numpy(), 1e-6, 0.0)
    x = torch.from_numpy(want)
    assert (x.abs() < 2.0 ** 128 * (1 - 2.0 ** -20)).all() and (x.abs() > 248 * 2.0 ** 120).any()
    # 2^-4, and the roundings of 32 bits on the way: 18 of the norm, 8 of the rotation (of the pair's size), 2^-24 each
    y = back[0].double()
    assert torch.isfinite(y).all()
    size = x.abs().amax(-1, keepdim=True) * 2
    assert ((y - x).abs() <= 2.0 ** -4 * x.abs() + 26 * 2.0 ** -24 * size + 2.0 ** 110).all()
    # and one token's attention gives the value as stored
    st1 = Q.Step(2, 2, d, [(0, 1)], 16, seed=4).upload()
    k1, v1 = torch.zeros(1, 2, d, device="cuda", dtype=torch.bfloat16), v[:1].contiguous()
    cfg1 = st1.config()
    B.tkphi_quant_append(cfg1, st1.step(), st1.pool(), B.make_new_rows(None, k1, v1, None), None, ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    out, _ = st1.call(B.tkphi_quant_attention, cfg1)
    assert np.array_equal(out[0], back[1, 0].double().numpy())
