"""tkphi_kv_append: rotated queries, pages and mean keys against the float64 oracle; everything else stays as it was."""
import numpy as np
import pytest
import torch

import paged_utils as P
from oracle import paged_oracle as O
from paper_2604_05438_amd import binding as B

pytestmark = pytest.mark.gpu


def inv_freq(rot):
    return 500000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))


def check_append(st, rot, adjacent, skip=(), with_q=True, in_place=False, status=0, freq=None, base=0):
    gen = torch.Generator().manual_seed(77)
    dt, d, G = P.dt(st.dtype), st.d, st.hq // st.hkv
    qkv = torch.randn(st.rows, st.hq + 2 * st.hkv, d, generator=gen).to(dt)
    dev = qkv.cuda()
    q, k, v = dev[:, :st.hq], dev[:, st.hq:st.hq + st.hkv], dev[:, st.hq + st.hkv:]
    q_rot = q if in_place else torch.full((st.rows, st.hq, d), 7.0, device="cuda", dtype=dt)
    freq = inv_freq(rot) if freq is None else freq
    f = torch.from_numpy(freq).cuda()
    st.upload()
    cfg, step, t = st.config(rot_dim=rot, rot_adjacent=adjacent), st.step(), st.dev
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    io = B.make_new_rows(q if with_q else None, k, v, q_rot if with_q else None, inv_freq=f if rot else None)
    B.tkphi_kv_append(cfg, step, B.make_pool(t["K"], t["V"], t["M"]), io, ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == status
    K, V = t["K"].double().cpu().numpy(), t["V"].double().cpu().numpy()
    wK, wV = P.f64(st.K).copy(), P.f64(st.V).copy()
    x, half, U = P.f64(qkv), P.HALF[st.dtype], P.U
    got_q = (qkv[:, :st.hq] if not with_q else q_rot).double().cpu().numpy()
    want_M = None if st.M is None else P.f64(st.M).copy()
    touched = np.zeros(st.rows, dtype=bool)

    def near(got, want, src):
        # sin and cos to 3 U, two products and a sum rounded once each: at most 6 U of the pair's size; then storage
        size = np.abs(src).max(-1, keepdims=True) * 2
        assert (np.abs(got - want) <= half * np.abs(want) * (1 + 2.0 ** -20) + 8 * U * size).all(), np.abs(got - want).max()

    for i, (n, m) in enumerate(st.lens):
        if i in skip:
            continue
        for j in range(m):
            row, pos = st.first[i] + j, n + j
            touched[row] = True
            p = st.table[i, pos // st.page] if pos // st.page < st.table.shape[1] else -1
            if with_q:
                near(got_q[row], O.rotate(x[row, :st.hq], pos, freq, adjacent), x[row, :st.hq])
            if 0 <= p < st.n_pages:
                near(K[p, :, pos % st.page], O.rotate(x[row, st.hq:st.hq + st.hkv], pos, freq, adjacent), x[row, st.hq:st.hq + st.hkv])
                assert np.array_equal(K[p, :, pos % st.page][..., rot:], x[row, st.hq:st.hq + st.hkv][..., rot:])
                wK[p, :, pos % st.page] = K[p, :, pos % st.page]
                wV[p, :, pos % st.page] = x[row, st.hq + st.hkv:]
        if st.block:
            for b in range(n // st.block, (n + m) // st.block):
                t0 = b * st.block
                p = st.table[i, t0 // st.page]
                if not 0 <= p < st.n_pages:
                    continue
                keys = K[p, :, t0 % st.page:t0 % st.page + st.block]
                at = t0 % st.page // st.block
                got = t["M"][p, :, at].double().cpu().numpy()
                want = keys.mean(1)
                assert (np.abs(got - want) <= half * np.abs(want) * (1 + 2.0 ** -20) + U * st.block * np.abs(keys).mean(1)).all()
                want_M[p, :, at] = got
    assert np.array_equal(K, wK) and np.array_equal(V, wV)           # nothing else moved
    if st.block:
        assert np.array_equal(t["M"].double().cpu().numpy(), want_M)
    if with_q and not in_place:
        assert (got_q[~touched] == 7).all()
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rot,adjacent", [(0, False), (16, False), (16, True), (64, False), (64, True), (-1, False), (-1, True)])
def test_rotations(dtype, d, rot, adjacent):
    st = P.Step(dtype, 6, 2, d, [(0, 1), (100000, 3), (15, 2), (7, 40)] if d == 64 else [(5, 1), (3, 30)], 16, seed=3)
    check_append(st, d if rot < 0 else rot, adjacent)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,block,heads_first", [(16, 16, True), (64, 16, False), (64, 64, True), (128, 32, False), (192, 64, True)])
def test_means_of_filled_blocks(dtype, page, block, heads_first):
    lens = [(0, 1), (block - 1, 1), (block - 2, 1), (5, block), (0, 3 * block + 1), (page - 1, 2), (block, 0), (2 * block - 3, 3)]
    check_append(P.Step(dtype, 4, 2, 64, lens, page, heads_first, block=block, seed=1), 64, False)
    check_append(P.Step(dtype, 8, 1, 128, lens, page, heads_first, block=block, seed=1), 128, True)


@pytest.mark.parametrize("page", [1, 7, 24, 100])
def test_odd_pages(page):
    check_append(P.Step("bf16", 14, 2, 64, [(3, 50), (0, 1), (99, 2)], page, heads_first=False, slack_rows=2), 32, True)


def test_keys_and_values_only_and_in_place():
    check_append(P.Step("bf16", 4, 2, 64, [(3, 20), (9, 1)], 16), 64, False, with_q=False)
    check_append(P.Step("bf16", 4, 2, 64, [(3, 20), (9, 1)], 16), 64, False, in_place=True)
    check_append(P.Step("f32", 4, 2, 64, [(3, 20), (9, 1)], 16), 32, True, in_place=True)


def test_far_positions_turn_exactly():
    """Angles of positions near 10^6 (in 32 bits they would be off by 0.06 rad), of any frequency."""
    freq = np.concatenate([[1.0, np.pi / 2, 3.0e3, 0.0, -1.0], 10.0 ** -np.arange(27)])
    st = P.Step("f32", 1, 1, 64, [(999_990, 12)], 4096)
    check_append(st, 64, False, freq=freq)


def test_many_sequences_and_other_row_order():
    r = np.random.default_rng(2)
    lens = [(int(r.integers(0, 40)), int(r.integers(0, 20))) for _ in range(130)]
    check_append(P.Step("bf16", 2, 1, 64, lens, 32, block=16, order=list(r.permutation(130)), slack_rows=5), 64, False)


def test_bad_descriptions_and_pages():
    lens = [(20, 1), (30, 2), (10, 7), (5, 1)]
    for i, word, value in ((1, 0, -1), (1, 1, -2), (2, 0, 1000), (2, 2, 6), (3, 2, -1)):
        st = P.Step("bf16", 4, 2, 64, lens, 16, block=16)
        st.seqs[i, word] = value
        check_append(st, 64, False, skip=(i,), status=B.TKPHI_DEV_BAD_LENGTH)
    for value in (-1, -7, 10 ** 9):
        st = P.Step("bf16", 4, 2, 64, lens, 16, block=16)
        st.table[2, 0] = value
        check_append(st, 64, False, status=B.TKPHI_DEV_BAD_PAGE)


@pytest.mark.parametrize("block", [0, 16])
def test_sequences_that_share_rows_do_no_harm(block):
    """More tiles than the rows allow for: what fits is written, the rest is left out and reported; nothing else moves."""
    st = P.Step("bf16", 4, 2, 64, [(0, 40)] * 30, 16, block=block, seed=1)
    st.seqs[:, 2] = 0
    st.rows = 40
    st.upload()
    qkv = torch.randn(40, 8, 64, generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    q_rot = torch.zeros(40, 4, 64, device="cuda", dtype=torch.bfloat16)
    cfg, step, t = st.config(rot_dim=0), st.step(), st.dev
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    B.tkphi_kv_append(cfg, step, B.make_pool(t["K"], t["V"], t["M"]), B.make_new_rows(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], q_rot), ws.data_ptr(), ws.numel(),
                      B.current_stream_ptr())
    assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == B.TKPHI_DEV_BAD_LENGTH
    assert torch.equal(q_rot, qkv[:, :4])
    for now, before, new in ((t["K"], st.K, qkv[:, 4:6]), (t["V"], st.V, qkv[:, 6:])):
        want = before.clone()
        done = 0
        for pages in st.table:
            for k in range(40):
                at = pages[k // 16], slice(None), k % 16
                got = now[at].cpu()
                if torch.equal(got, new[k].cpu()):
                    want[at] = got
                    done += 1
        assert torch.equal(now.cpu(), want) and 40 <= done < 30 * 40
