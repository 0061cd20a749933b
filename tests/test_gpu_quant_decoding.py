"""What every code and scale byte stands for: the bf16 number nearest to code x 2^(b - 127)."""
import pytest
import torch

import paged_utils as P
import quant_utils as Q
from paper_2604_05438_amd import binding as B

pytestmark = pytest.mark.gpu


def every_code(b):
    """A step whose tokens hold all codes with the scale bytes b, two rows each; codes and bytes by token"""
    n = 2 * len(b)
    st = Q.Step(1, 1, 128, [(0, n)], 16)
    t = torch.arange(n)
    page = torch.from_numpy(st.table[0].copy()).long()[t // 16]
    codes = ((t % 2)[:, None] * 128 + torch.arange(128)[None]).to(torch.uint8)
    bytes_ = torch.tensor(b, dtype=torch.uint8)[t // 2]
    for x in (st.K8, st.V8):
        x.view(torch.uint8)[page, 0, t % 16] = codes
    st.S[page, 0, t % 16] = bytes_[:, None].expand(n, 2)
    st.take_values()
    return st.upload(), codes.view(torch.float8_e4m3fn), bytes_


def read(st):
    cfg, step = st.config(), st.step()
    out = torch.empty(2, st.rows, 1, 128, device="cuda", dtype=torch.bfloat16)
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    B.tkphi_quant_read(cfg, step, st.pool(), B.make_read_rows(out[0], out[1]), ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == 0
    return out.cpu()[:, :, 0]


def test_rows_of_every_code_and_scale():
    st, codes, b = every_code(range(1, 255))
    exact = codes.double() * torch.exp2(b.double() - 127)[:, None]       # (a number of 32 bits, or past them)
    want = exact.bfloat16()
    for got in read(st):
        wrong = ~(torch.isnan(want) & torch.isnan(got)) & (got != want)
        assert not wrong.any(), [(int(b[i]), float(codes[i, c]), float(got[i, c]), float(want[i, c])) for i, c in wrong.nonzero()[:8].tolist()]
    inside = ((b >= 3) & (b <= 246))[:, None] & ~torch.isnan(exact)
    assert (want.double()[inside.expand_as(exact)] == exact[inside.expand_as(exact)]).all()      # what the documentation calls exact
    for byte in (1, 2, 247):
        assert not torch.equal(want[b == byte].double().nan_to_num(0, 9e99, -9e99), exact[b == byte].nan_to_num(0, 9e99, -9e99))


@pytest.mark.parametrize("rows", [1, 40])
def test_values_of_every_code_and_scale_in_attention(rows):
    """A token that only it sees itself gives its value back, from the split kernel and the chunk kernel (a window of one token)"""
    st, codes, b = every_code(list(range(1, 255)))
    n = 2 * 254
    lens = [(t, min(rows, n - t)) for t in range(0, n, rows)]
    st.seqs = torch.tensor([[t, m, t, 0] for t, m in lens], dtype=torch.int32).cuda()
    st.K8.view(torch.uint8).zero_()
    st.dev["K8"].view(torch.uint8).zero_()
    pages = st.dev["pages"].expand(len(lens), -1).contiguous()
    step = B.make_step(st.seqs, pages, n, max(m for _, m in lens), n)
    cfg = st.config(window=1)
    out = torch.empty(n, 1, 128, device="cuda", dtype=torch.bfloat16)
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    B.tkphi_quant_attention(cfg, step, st.pool(), B.make_attention_rows(st.dev["q"], out, None), ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == 0
    want, got = (codes.double() * torch.exp2(b.double() - 127)[:, None]).bfloat16(), out.cpu()[:, 0]
    assert (torch.isnan(got) == torch.isnan(want)).all()
    # (below the least number of full precision the matrix instructions may give 0)
    there = ~torch.isnan(want) & (want.abs().double() >= 2.0 ** -126)
    assert torch.equal(got[there], want[there]) and (got[~there & ~torch.isnan(want)].abs().double() <= 2.0 ** -126).all()
