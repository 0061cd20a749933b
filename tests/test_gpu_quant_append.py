"""tkphi_norm_append, tkphi_quant_append and tkphi_quant_read: normed and rotated heads, codes, scales and mean keys against the float64 oracle; everything
else stays as it was."""
import numpy as np
import pytest
import torch

import paged_utils as P
import quant_utils as Q
from oracle import paged_oracle as O
from paper_2604_05438_amd import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-5


def inv_freq(rot):
    return 500000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))


def weights(st, kind, offset, seed=5):
    """(device, float64) weights of queries and keys: shared by all heads, one row per head, or none"""
    gen = torch.Generator().manual_seed(seed)
    dev, ref = [], []
    for h in (st.hq, st.hkv):
        w = (torch.rand(h, st.d, generator=gen) + 0.5 - offset).to(P.dt(st.dtype))
        w = {"shared": w[:1], "heads": w, "ones": None}[kind]
        dev.append(None if w is None else w[0].cuda() if kind == "shared" else w.cuda())
        ref.append(None if w is None else P.f64(w))
    return dev, ref


def check(st, rot, adjacent=False, norm="shared", offset=0.0, eps=EPS, skip=(), with_q=True, status=0, change=None):
    """norm: kind of weights, or None.  change(qkv): the inputs, before they are used."""
    quant = isinstance(st, Q.Step)
    gen = torch.Generator().manual_seed(77)
    dt, d = P.dt(st.dtype), st.d
    qkv = torch.randn(st.rows, st.hq + 2 * st.hkv, d, generator=gen).to(dt)
    if change:
        change(qkv)
    dev = qkv.cuda()
    q, k, v = dev[:, :st.hq], dev[:, st.hq:st.hq + st.hkv], dev[:, st.hq + st.hkv:]
    q_rot = torch.full((st.rows, st.hq, d), 7.0, device="cuda", dtype=dt)
    freq = inv_freq(rot)
    f = torch.from_numpy(freq).cuda()
    st.upload()
    cfg, step, t = st.config(rot_dim=rot, rot_adjacent=adjacent), st.step(), st.dev
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    io = B.make_new_rows(q if with_q else None, k, v, q_rot if with_q else None, inv_freq=f if rot else None)
    (qw, kw), (qr, kr) = weights(st, norm, offset) if norm else ((None, None), (None, None))
    norms = B.make_head_norms(qw, kw, eps, offset) if norm else None
    if quant:
        B.tkphi_quant_append(cfg, step, st.pool(), io, norms, ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    else:
        B.tkphi_norm_append(cfg, step, B.make_pool(t["K"], t["V"], t["M"]), io, norms, ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == status
    x, half, U = P.f64(qkv), P.HALF[st.dtype], P.U
    # the mean square is a chain of at most 2 x 8 sums per lane and 4 across lanes, each rounding by U, its root and what it multiplies by 2 U and U each; w + offset U
    chain = (24 / 2 + 6) * U if norm else 0.0

    def turned(row, heads, w, pos):
        y = x[row, heads]
        if norm:
            y = O.head_norm(y, w, eps, offset)
        return y, O.rotate(y, pos, freq, adjacent)

    def size(y):
        # sin and cos to 3 U, two products and a sum rounded once each: at most 6 U of the pair's size, of values that the norm has off by `chain`
        # (an element that is finite comes out of finite ones: those that are not take no part in its error)
        return (8 * U + chain) * 2 * np.abs(np.where(np.isfinite(y), y, 0.0)).max(-1, keepdims=True)
    if quant:
        codes = {n: t[n + "8"].cpu() for n in "KV"}
        S = t["S"].cpu().numpy()
        wS = st.S.numpy().copy()
        got = {n: P.f64(codes[n]) for n in "KV"}
        want = {n: P.f64(getattr(st, n + "8")).copy() for n in "KV"}
    else:
        got = {n: t[n].double().cpu().numpy() for n in "KV"}
        want = {n: P.f64(getattr(st, n)).copy() for n in "KV"}
    want_M = None if st.M is None else P.f64(st.M).copy()
    q_got = q_rot.double().cpu().numpy()
    touched = np.zeros(st.rows, dtype=bool)
    for i, (n, m) in enumerate(st.lens):
        if i in skip:
            continue
        for j in range(m):
            row, pos = st.first[i] + j, n + j
            touched[row] = True
            p, at = st.table[i, pos // st.page] if pos // st.page < st.table.shape[1] else -1, pos % st.page
            if with_q:
                y, w = turned(row, slice(0, st.hq), qr, pos)
                assert (np.abs(q_got[row] - w) <= half * np.abs(w) * (1 + 2.0 ** -20) + size(y)).all(), (i, j)
            if not 0 <= p < st.n_pages:
                continue
            y, w = turned(row, slice(st.hq, st.hq + st.hkv), kr, pos)
            v_row = x[row, st.hq + st.hkv:]
            if not quant:
                assert (np.abs(got["K"][p, :, at] - w) <= half * np.abs(w) * (1 + 2.0 ** -20) + size(y)).all(), (i, j)
                want["K"][p, :, at], want["V"][p, :, at] = got["K"][p, :, at], v_row
                continue
            vc, vb = O.quantise(v_row)
            want["V"][p, :, at], wS[p, :, at, 1] = vc, vb                     # (nothing is computed on the way: to the bit)
            kc, kb = O.quantise(w)
            step_up = np.exp2(S[p, :, at, 0].astype(np.int64) - 127.0)[:, None]
            # the scale: another one only where the largest element is within the arithmetic's error of 448 times a power
            top = np.abs(w).max(-1)
            for h in range(st.hkv):
                if S[p, h, at, 0] != kb[h]:
                    edge = 448 * np.exp2(min(S[p, h, at, 0], kb[h]) - 127.0)
                    assert abs(int(S[p, h, at, 0]) - int(kb[h])) == 1 and abs(top[h] - edge) <= size(y)[h, 0], (i, j, h)
            err = np.abs(got["K"][p, :, at] * step_up - w)
            bound = np.maximum(2.0 ** -4 * np.abs(w), 2.0 ** -10 * step_up) * (1 + 2.0 ** -20) + size(y) * (1 + 2.0 ** -4)
            assert (err <= bound)[np.isfinite(w)].all(), (i, j, (err / bound).max())
            assert np.isnan(got["K"][p, :, at][~np.isfinite(w)]).all()
            want["K"][p, :, at], wS[p, :, at, 0] = got["K"][p, :, at], S[p, :, at, 0]
        if st.block:
            for b in range(n // st.block, (n + m) // st.block):
                t0 = b * st.block
                p = st.table[i, t0 // st.page]
                if not 0 <= p < st.n_pages:
                    continue
                here = p, slice(None), slice(t0 % st.page, t0 % st.page + st.block)
                keys = got["K"][here] * (np.exp2(S[here][..., 0] - 127.0)[..., None] if quant else 1.0)
                at = t0 % st.page // st.block
                M = t["M"][p, :, at].double().cpu().numpy()
                mean = keys.mean(1)
                assert (np.abs(M - mean) <= half * np.abs(mean) * (1 + 2.0 ** -20) + U * st.block * np.abs(keys).mean(1)).all()
                want_M[p, :, at] = M
    for n in "KV":
        assert np.array_equal(got[n], want[n], equal_nan=True), n             # nothing else moved
    if quant:
        assert np.array_equal(S, wS)
    if st.block:
        assert np.array_equal(t["M"].double().cpu().numpy(), want_M, equal_nan=True)
    assert (q_got[~touched] == 7).all()


# ---- norms --------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rot,adjacent", [(0, False), (16, True), (64, False), (-1, False), (-1, True)])
@pytest.mark.parametrize("norm,offset", [("shared", 0.0), ("heads", 1.0), ("ones", 0.0)])
def test_norms(dtype, d, rot, adjacent, norm, offset):
    st = P.Step(dtype, 6, 2, d, [(0, 1), (100000, 3), (15, 2), (7, 40)] if d == 64 else [(5, 1), (3, 30)], 16, seed=3)
    check(st, d if rot < 0 else rot, adjacent, norm, offset)


def test_norms_with_means_odd_pages_and_keys_only():
    lens = [(0, 1), (15, 1), (14, 1), (5, 16), (0, 49), (63, 2), (16, 0), (29, 3)]
    check(P.Step("bf16", 4, 2, 64, lens, 64, block=16, seed=1), 64)
    check(P.Step("f32", 8, 1, 128, lens, 64, False, block=16, seed=1), 128, True)
    check(P.Step("bf16", 14, 2, 64, [(3, 50), (0, 1), (99, 2)], 7, heads_first=False, slack_rows=2), 32, True)
    check(P.Step("bf16", 4, 2, 64, [(3, 20), (9, 1)], 16), 64, with_q=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norms_of_small_and_large_heads(dtype):
    """Rows of zeros come out as zeros; rows whose squares are far below eps, and far above it"""
    def sizes(qkv):
        qkv[0] = 0
        qkv[1] *= 1e-9
        qkv[2] *= 1e15
    check(P.Step(dtype, 4, 2, 128, [(3, 6)], 16), 128, change=sizes)
    check(P.Step(dtype, 4, 2, 64, [(3, 6)], 16), 64, change=sizes, eps=1e-30)


# ---- the cache in 8 bits ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rot,adjacent", [(0, False), (16, False), (16, True), (64, True), (-1, False), (-1, True)])
@pytest.mark.parametrize("norm", [None, "shared"])
def test_codes(d, rot, adjacent, norm):
    st = Q.Step(6, 2, d, [(0, 1), (100000, 3), (15, 2), (7, 40)] if d == 64 else [(5, 1), (3, 30)], 16, seed=3)
    check(st, d if rot < 0 else rot, adjacent, norm)


@pytest.mark.parametrize("page,block,heads_first", [(16, 16, True), (64, 16, False), (64, 64, True), (128, 32, False), (192, 64, True)])
def test_codes_and_means_of_filled_blocks(page, block, heads_first):
    lens = [(0, 1), (block - 1, 1), (block - 2, 1), (5, block), (0, 3 * block + 1), (page - 1, 2), (block, 0), (2 * block - 3, 3)]
    check(Q.Step(4, 2, 64, lens, page, heads_first, block=block, seed=1), 64, norm=None)
    check(Q.Step(8, 1, 128, lens, page, heads_first, block=block, seed=1), 128, True)


@pytest.mark.parametrize("page", [1, 7, 24, 100])
def test_codes_on_odd_pages(page):
    check(Q.Step(14, 2, 64, [(3, 50), (0, 1), (99, 2)], page, heads_first=False, slack_rows=2), 32, True, norm=None)


def test_codes_of_keys_and_values_only():
    check(Q.Step(4, 2, 64, [(3, 20), (9, 1)], 16), 64, with_q=False, norm=None)


def test_codes_at_the_borders():
    """Rows of zeros, of one element, with the largest element at, just below and just above 448 and 464 times a power of two, ties between codes, subnormal codes, the
    smallest and largest numbers, infinities and NaN"""
    def borders(qkv):
        kv = qkv[:, 4:]
        kv[0] = 0
        kv[1] = 0
        kv[1, :, 5] = -3.0
        for i, top in enumerate((448.0, 446.0, 450.0, 464.0, 466.0, 256.0, 255.0, 512.0)):
            kv[2 + i] = kv[2 + i].clamp(-1, 1) * 100
            kv[2 + i, :, 9] = top * 2.0 ** (i - 3)
        kv[10] = torch.linspace(-1, 1, 64) * 15.5            # ties among others
        kv[10, :, 0] = 448
        kv[11] *= 2.0 ** -11
        kv[11, :, 0] = 448
        kv[12] *= 1e-38
        kv[13] *= 1e-36
        kv[14] *= 3e37
        kv[15, :, 3] = float("inf")
        kv[16, :, 4] = float("nan")
        kv[17, :] = float("-inf")
        kv[18, :, ::2] = float("nan")
        kv[19, :, 0] = float("nan")
        kv[19, :, 1:] = 0
    check(Q.Step(4, 2, 64, [(0, 20)], 16), 0, norm=None, change=borders)


def test_codes_of_bad_descriptions_and_pages():
    lens = [(20, 1), (30, 2), (10, 7), (5, 1)]
    for i, word, value in ((1, 0, -1), (1, 1, -2), (2, 0, 1000), (2, 2, 6), (3, 2, -1)):
        st = Q.Step(4, 2, 64, lens, 16, block=16)
        st.seqs[i, word] = value
        check(st, 64, skip=(i,), status=B.TKPHI_DEV_BAD_LENGTH)
    for value in (-1, -7, 10 ** 9):
        st = Q.Step(4, 2, 64, lens, 16, block=16)
        st.table[2, 0] = value
        check(st, 64, norm=None, status=B.TKPHI_DEV_BAD_PAGE)


def test_codes_of_many_sequences_in_another_order_of_rows():
    r = np.random.default_rng(2)
    lens = [(int(r.integers(0, 40)), int(r.integers(0, 20))) for _ in range(130)]
    check(Q.Step(2, 1, 64, lens, 32, block=16, order=list(r.permutation(130)), slack_rows=5), 64)


@pytest.mark.parametrize("d", [64, 128])
def test_queries_in_place(d):
    """q_rot may be q itself: the same as in rows of their own, with norms and codes"""
    st = Q.Step(6, 2, d, [(3, 20), (9, 1)], 16).upload()
    qkv = torch.randn(st.rows, 10, d, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    q_rot = torch.empty(st.rows, 6, d, device="cuda", dtype=torch.bfloat16)
    freq, weight = torch.from_numpy(inv_freq(d)).cuda(), torch.full((d,), 0.75, device="cuda", dtype=torch.bfloat16)
    cfg, step, norms = st.config(rot_dim=d), st.step(), B.make_head_norms(weight, weight, EPS)
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    for out in (q_rot, qkv[:, :6]):
        io = B.make_new_rows(qkv[:, :6], qkv[:, 6:8], qkv[:, 8:], out, inv_freq=freq)
        B.tkphi_quant_append(cfg, step, st.pool(), io, norms, ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    torch.cuda.synchronize()
    assert torch.equal(qkv[:, :6], q_rot)


# ---- read back ------------------------------------------------------------------------------------------------------------------------
def read(st, status=0, layout="rows", want_k=True, want_v=True):
    """Every row of the step against what its token's codes stand for; the others stay 7"""
    st.upload()
    shape = (st.rows, st.hkv, st.d) if layout == "rows" else (st.hkv, st.rows, st.d)
    out = [torch.full(shape, 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    views = [x if layout == "rows" else x.transpose(0, 1) for x in out]
    cfg, step = st.config(), st.step()
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    io = B.make_read_rows(views[0] if want_k else None, views[1] if want_v else None)
    B.tkphi_quant_read(cfg, step, st.pool(), io, ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == status
    for x, pool, wanted in ((views[0], st.K, want_k), (views[1], st.V, want_v)):
        want = torch.full((st.rows, st.hkv, st.d), 7.0, dtype=torch.bfloat16)
        if wanted:
            for i, (n, m) in enumerate(st.lens):
                if not 0 <= st.seqs[i, 0] < 10 ** 5:
                    continue
                for j in range(m):
                    p = st.table[i, (n + j) // st.page]
                    want[st.first[i] + j] = pool[p, :, (n + j) % st.page] if 0 <= p < st.n_pages else 0.0
        assert torch.equal(x.cpu().nan_to_num(9.0), want.nan_to_num(9.0))


@pytest.mark.parametrize("heads,page,heads_first", [((4, 2, 64), 16, True), ((8, 1, 128), 64, False), ((24, 8, 128), 100, True), ((14, 2, 64), 7, False), ((3, 3, 64), 256, True)])
@pytest.mark.parametrize("layout", ["rows", "heads"])
def test_read_back(heads, page, heads_first, layout):
    read(Q.Step(*heads, [(0, 1), (63, 1), (64, 2), (0, 64), (5, 130), (40, 0), (61, 67)], page, heads_first, seed=4, slack_rows=3), layout=layout)


def test_read_keys_or_values_only_and_bad_pages():
    read(Q.Step(4, 2, 64, [(3, 70)], 16), want_k=False)
    read(Q.Step(4, 2, 64, [(3, 70)], 16), want_v=False)
    for value in (-1, -7, 10 ** 9):
        st = Q.Step(4, 2, 64, [(3, 70), (0, 5)], 16)
        st.table[0, 2] = value
        read(st, status=B.TKPHI_DEV_BAD_PAGE)
    st = Q.Step(4, 2, 64, [(3, 70), (0, 5)], 16)
    st.seqs[1, 0] = 10 ** 6
    read(st, status=B.TKPHI_DEV_BAD_LENGTH)
    st = Q.Step(4, 2, 64, [(0, 30)], 16, change=lambda s: s.K.view(-1)[::77].fill_(float("nan")))
    read(st)


def test_read_of_sequences_that_share_rows_does_no_harm():
    st = Q.Step(4, 2, 64, [(0, 200)] * 30, 16, seed=1)
    st.seqs[:, 2] = 0
    st.rows, st.q = 200, st.q[:200]
    st.upload()
    out = torch.full((200, 2, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    cfg, step = st.config(), st.step()
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    B.tkphi_quant_read(cfg, step, st.pool(), B.make_read_rows(out, None), ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == B.TKPHI_DEV_BAD_LENGTH
    assert torch.isfinite(out).all()
