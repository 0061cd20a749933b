"""Norms of heads at the ends of 32 bits: squares that sum to less than 2^128 are normed, those beyond come out as zeros, in rows, codes and read back."""
import numpy as np
import pytest
import torch

import paged_utils as P
import quant_utils as Q
from oracle import paged_oracle as O
from paper_2604_05438_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f32", "codes"])
@pytest.mark.parametrize("d", [64, 128])
def test_heads_whose_squares_overflow(kind, d):
    dtype = "f32" if kind == "f32" else "bf16"
    st = (Q.Step(2, 1, d, [(0, 4)], 16, seed=2) if kind == "codes" else P.Step(dtype, 2, 1, d, [(0, 4)], 16, seed=2)).upload()
    x = torch.randn(4, 4, d, generator=torch.Generator().manual_seed(1)).clamp(-3, 3) * torch.tensor([1.0, 2.0 ** 58, 2.0 ** 70, 2.0 ** 100])[:, None, None]
    x = x.to(P.dt(dtype))                                    # (9 x 128 x 2^116 < 2^127; at 2^70 one square is beyond)
    x[2:, :, 0] = x[2:, :, 0].abs() + 2.0 ** 70
    dev, q_rot = x.cuda(), torch.full((4, 2, d), 7.0, device="cuda", dtype=P.dt(dtype))
    cfg, step, t = st.config(), st.step(), st.dev
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    io, norms = B.make_new_rows(dev[:, :2], dev[:, 2:3], dev[:, 3:], q_rot), B.make_head_norms(None, None, 1e-6)
    call, pool = (B.tkphi_quant_append, st.pool()) if kind == "codes" else (B.tkphi_norm_append, B.make_pool(t["K"], t["V"], t["M"]))
    call(cfg, step, pool, io, norms, ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == 0
    page = int(st.table[0, 0])
    K = (t["K8"].double() * torch.exp2(t["S"][..., 0].double() - 127)[..., None] if kind == "codes" else t["K"].double())[page, :, :4].transpose(0, 1).cpu().numpy()
    want = O.head_norm(x.double().numpy(), None, 1e-6, 0.0)
    want[2:] = 0
    # 18 roundings of 32 bits, half a step of what is stored, half the least code
    near = (18 * 2.0 ** -24 + P.HALF[dtype]) * np.abs(want) * (1 + 2.0 ** -20)
    assert (np.abs(q_rot.double().cpu().numpy() - want[:, :2]) <= near[:, :2]).all()
    if kind == "codes":
        near = np.maximum(2.0 ** -4 * np.abs(want) * (1 + 2.0 ** -18), np.where(want == 0, 0.0, 2.0 ** -10 * 2.0 ** -6))
        assert (t["S"][page, 0, 2:4, 0] == 10).all()
    assert (np.abs(K - want[:, 2:3]) <= near[:, 2:3]).all()
