"""tkphi_quant_attention and tkphi_quant_block_attention against the float64 oracle over the values that the codes stand for, with the bounds of a bf16 cache."""
import numpy as np
import pytest
import torch

import paged_utils as P
import quant_utils as Q
from paper_2604_05438_amd import binding as B

pytestmark = pytest.mark.gpu

HEADS = {"1b": (32, 8, 64), "3b": (24, 8, 128), "one": (1, 1, 64), "wide": (8, 1, 128), "odd": (14, 2, 64), "five": (10, 2, 128), "mha": (3, 3, 64)}


def run(model, lens, page, window=0, workgroups=0, scale=None, **kw):
    st = Q.Step(*HEADS[model], lens, page, **kw).upload()
    cfg = st.config(window=window, workgroups=workgroups, **({} if scale is None else {"scale": scale}))
    out, lse = st.call(B.tkphi_quant_attention, cfg)
    P.check(st, out, lse, P.attention_oracle(st, scale=scale, window=window))
    return st


@pytest.mark.parametrize("model", list(HEADS))
def test_single_tokens(model):
    """From a lone token to some hundreds, across tile and page ends."""
    run(model, [(0, 1), (1, 1), (14, 1), (15, 1), (16, 1), (31, 1), (127, 1), (128, 1), (500, 1)], 16)


@pytest.mark.parametrize("page,heads_first", [(1, True), (7, False), (8, True), (24, True), (64, False), (100, True), (256, False)])
@pytest.mark.parametrize("model", ["odd", "five"])
def test_pages_and_orders(model, page, heads_first):
    run(model, [(77, 1), (0, 3), (300, 2), (255, 1)], page, heads_first=heads_first)


@pytest.mark.parametrize("model", ["one", "3b", "wide", "odd"])
@pytest.mark.parametrize("lens", [[(40, 5)], [(0, 17), (33, 4), (100, 1)], [(0, 70), (61, 40), (5, 0), (200, 3)], [(130, 150)]])
def test_chunks(model, lens):
    run(model, lens, 16)


@pytest.mark.parametrize("page,heads_first", [(1, True), (7, False), (24, True), (64, False), (100, True)])
@pytest.mark.parametrize("model", ["odd", "five"])
def test_chunks_on_pages(model, page, heads_first):
    run(model, [(77, 60), (0, 130)], page, heads_first=heads_first)


@pytest.mark.parametrize("window", [1, 5, 64, 129])
@pytest.mark.parametrize("lens", [[(300, 1), (3, 1), (64, 1)], [(0, 90), (200, 33)]])
@pytest.mark.parametrize("model", ["odd", "five"])
def test_windows(model, window, lens):
    run(model, lens, 24, window=window)


@pytest.mark.parametrize("workgroups", [1, 2, 3, 7, 40, 333])
@pytest.mark.parametrize("model", ["odd", "five"])
def test_work_cut_anywhere(model, workgroups):
    """Items whole, shared by several workgroups, several items per workgroup; single tokens and chunks."""
    run(model, [(900, 1), (5, 1), (2000, 2), (0, 1)], 32, workgroups=workgroups)
    run(model, [(700, 40), (0, 90), (64, 1)], 32, workgroups=workgroups, seed=3)


def test_many_sequences():
    r = np.random.default_rng(5)
    run("one", [(int(r.integers(0, 60)), int(r.integers(0, 3))) for _ in range(150)], 16, slack_rows=3)
    run("five", [(int(r.integers(0, 90)), int(r.integers(0, 12))) for _ in range(90)], 16, slack_rows=1)


@pytest.mark.parametrize("model,workgroups", [("one", 1), ("1b", 3), ("odd", 2), ("five", 7)])
@pytest.mark.parametrize("heads_first", [True, False])
def test_many_sequences_with_much_work_per_workgroup(model, workgroups, heads_first):
    r = np.random.default_rng(7)
    lens = [(int(r.integers(0, 300)), int(r.integers(0, 2))) for _ in range(70)] + [(900, 1)]
    run(model, lens, 16, workgroups=workgroups, heads_first=heads_first, garbage=float("nan"), slack_rows=1)
    run(model, lens, 16, workgroups=workgroups, heads_first=heads_first, window=50)


def spread_scales(st):
    """Rows whose sizes differ by powers of ten, in keys and values"""
    gen = torch.Generator().manual_seed(9)
    for x in (st.K, st.V):
        x *= (10.0 ** (torch.rand(x.shape[:3], generator=gen) * 6 - 4))[..., None].to(x.dtype)


@pytest.mark.parametrize("model", ["odd", "five"])
@pytest.mark.parametrize("lens", [[(400, 1), (30, 2)], [(200, 50), (0, 33)]])
def test_rows_of_very_different_sizes(model, lens):
    run(model, lens, 16, change=spread_scales, scale=0.02)


@pytest.mark.parametrize("lens", [[(37, 1), (0, 1), (150, 3)], [(37, 40), (0, 33)]])
@pytest.mark.parametrize("model", ["odd", "five"])
@pytest.mark.parametrize("byte", [0, 255, None])
def test_what_nobody_sees_may_hold_anything(model, lens, byte):
    """Codes that are no numbers, and scale bytes that stand for nothing, behind the ends and in pages of nobody"""
    for page, window in ((32, 0), (100, 20)):
        st = Q.Step(*HEADS[model], lens, page, garbage=float("nan"), seed=7)
        want = P.attention_oracle(st, window=window)
        if byte is not None:
            nobody = torch.isnan(st.K).any(-1)
            st.S[nobody] = byte
        st.upload()
        out, lse = st.call(B.tkphi_quant_attention, st.config(window=window))
        P.check(st, out, lse, want)


@pytest.mark.parametrize("model", ["odd", "five"])
@pytest.mark.parametrize("lens,token,window", [([(50, 30)], 60, 0), ([(0, 120)], 60, 20), ([(58, 4)], 60, 0), ([(60, 1)], 60, 0)])
@pytest.mark.parametrize("what", ["V", "K", "overflow"])
def test_later_tokens_do_not_touch_earlier_queries(model, lens, token, window, what):
    """A code of token 60 that is no number, or a value that its scale makes infinite: the queries before it do not notice"""
    hq, hkv, d = HEADS[model]

    def change(st):
        if what != "overflow":
            getattr(st, what)[st.table[0, token // 16], 1, token % 16, 5] = float("nan")
    st = Q.Step(hq, hkv, d, lens, 16, seed=8, change=change)
    if what == "overflow":
        st.V8[st.table[0, token // 16], 1, token % 16, 5] = 448.0
        st.S[st.table[0, token // 16], 1, token % 16, 1] = 254
        st.take_values()
        assert not np.isfinite(P.f64(st.V)).all()
    st.upload()
    out, lse = st.call(B.tkphi_quant_attention, st.config(window=window))
    want = P.attention_oracle(st, window=window)
    n, G = lens[0][0], hq // hkv
    for i in range(lens[0][1]):
        clean = n + i < token or (window and n + i >= token + window)
        for g in range(hq if clean else G):
            by, bl = P.bounds("bf16", d, n + i + 1, *want[0][i][g])
            assert (np.abs(out[i, g] - want[0][i][g][0]) <= by).all() and abs(lse[i, g] - want[0][i][g][1]) <= bl, (i, g)
        if not clean and what != "K":
            assert not np.isfinite(out[i, G:, 5]).any()


@pytest.mark.parametrize("model,lens", [("odd", [(1500, 2), (1100, 1), (5, 1)]), ("one", [(4000, 1)]), ("1b", [(1027, 2), (0, 1)])])
@pytest.mark.parametrize("page", [16, 56])
def test_single_tokens_of_64_channels_with_much_work_per_workgroup(model, lens, page):
    """64 tokens at a time: absent pages, garbage that nobody sees, a value and a scale that are no numbers, windows"""
    hq, hkv, d = HEADS[model]
    for case in ("plain", "absent", "garbage", "overflow", "window"):
        window = 700 if case == "window" else 0
        st = Q.Step(hq, hkv, d, lens, page, seed=8, garbage=float("nan") if case == "garbage" else None)
        if case == "absent":
            st.table[0, [1, 2, 5]] = -1
        token = lens[0][0]                       # the first new token of the first sequence; later ones, if there are any, see it
        if case == "overflow":
            at = st.table[0, token // page], hkv - 1, token % page
            st.V8[(*at, 5)] = 448.0
            st.S[(*at, 1)] = 254
            st.take_values()
        want = P.attention_oracle(st, window=window)
        if case == "garbage":
            st.S[torch.isnan(st.K).any(-1)] = 255
        st.upload()
        out, lse = st.call(B.tkphi_quant_attention, st.config(workgroups=1, window=window))
        P.check(st, out, lse, want)


PAIRS = {"1b": (32, 8, 64), "odd": (14, 2, 64), "mha": (4, 4, 64), "wide": (16, 2, 64)}


@pytest.mark.parametrize("model,lens", [("1b", [(0, 1), (1, 1), (31, 1), (500, 1), (2000, 2), (63, 2)]), ("odd", [(0, 1), (15, 1), (127, 1), (1500, 1)]),
                                        ("mha", [(0, 8), (100, 5), (7, 1), (900, 3), (3, 0)]), ("wide", [(700, 1), (64, 1)])])
@pytest.mark.parametrize("page,workgroups", [(16, 0), (8, 1), (104, 3), (64, 40)])
def test_two_heads_that_adjoin(model, lens, page, workgroups):
    """Tokens outermost and 64 channels: heads by twos.  Absent pages, garbage, windows; codes of the one head that are no numbers do not touch the other's rows."""
    hq, hkv, d = PAIRS[model]
    for case in ("plain", "absent", "garbage", "window", "V", "K"):
        window = 40 if case == "window" else 0
        st = Q.Step(hq, hkv, d, lens, page, heads_first=False, seed=8, garbage=float("nan") if case == "garbage" else None, slack_rows=1)
        if case == "absent":
            st.table[-1, 0] = -1
        if case in "VK":
            n, m = lens[-1]
            st_at = st.table[-1, n // page], n % page
            getattr(st, case + "8")[st_at[0], 1, st_at[1], 5] = float("nan")
            if m:
                st.take_values()
        want = P.attention_oracle(st, window=window)
        if case == "garbage":
            st.S[torch.isnan(st.K).any(-1)] = 255
        st.upload()
        cfg = st.config(workgroups=workgroups, window=window)
        assert (cfg.stride_head, cfg.stride_tok) == (64, 64 * hkv)
        out, lse = st.call(B.tkphi_quant_attention, cfg)
        if case == "K":                          # rows of the head itself: the NaN's weight, and so what comes out, is undefined where the token is seen
            G = hq // hkv
            for g in range(hq):
                if g // G != 1:
                    for i, (n, m) in enumerate(lens):
                        for k in range(m):
                            by, bl = P.bounds("bf16", d, n + m, *want[i][k][g])
                            assert (np.abs(out[st.first[i] + k, g] - want[i][k][g][0]) <= by).all() and abs(lse[st.first[i] + k, g] - want[i][k][g][1]) <= bl
        else:
            P.check(st, out, lse, want)


def test_absent_pages_are_seen_by_nobody():
    for model in ("odd", "five"):
        lens = [(100, 1), (40, 30), (30, 1), (3, 2)]
        st = Q.Step(*HEADS[model], lens, 16, seed=2)
        st.table[0, 2] = -1
        st.table[1, [0, 3]] = -1
        st.table[2, :] = -1               # nothing at all: 0 and -inf
        st.table[3, 0] = -1
        st.upload()
        out, lse = st.call(B.tkphi_quant_attention, st.config())
        P.check(st, out, lse, P.attention_oracle(st))
        assert (out[st.first[2]] == 0).all() and np.isneginf(lse[st.first[2]]).all()
        st = Q.Step(*HEADS[model], [(100, 1), (90, 20)], 16, seed=2)
        st.table[0, 5:] = -1
        st.table[1, :] = -1
        st.upload()
        out, lse = st.call(B.tkphi_quant_attention, st.config(window=10))
        P.check(st, out, lse, P.attention_oracle(st, window=10))


def test_bad_descriptions_are_skipped_and_reported():
    lens = [(20, 1), (30, 2), (10, 1), (5, 1), (6, 1)]
    for i, word, value in ((1, 0, -1), (1, 1, -2), (2, 0, 1000), (2, 2, 6), (3, 2, -1), (4, 1, 3)):
        st = Q.Step(14, 2, 64, lens, 16)
        st.seqs[i, word] = value
        st.upload()
        out, lse = st.call(B.tkphi_quant_attention, st.config(), check_status=B.TKPHI_DEV_BAD_LENGTH)
        P.check(st, out, lse, P.attention_oracle(st), skip=(i,))
    for value in (-2, 10 ** 9, 14):
        st = Q.Step(14, 2, 64, lens, 16)
        st.table[0, 1] = value if value != 14 else st.n_pages
        st.upload()
        out, lse = st.call(B.tkphi_quant_attention, st.config(), check_status=B.TKPHI_DEV_BAD_PAGE)
        P.check(st, out, lse, P.attention_oracle(st))


@pytest.mark.parametrize("model", ["odd", "five"])
@pytest.mark.parametrize("lens", [[(3000, 1), (70, 2)], [(1000, 64), (5, 40)]])
def test_a_mean_of_equal_values_is_that_value(model, lens):
    def ones(st):
        st.V[:] = 1.0
    st = Q.Step(*HEADS[model], lens, 16, seed=11, change=ones).upload()
    out, lse = st.call(B.tkphi_quant_attention, st.config())
    assert (out == 1.0).all()


@pytest.mark.parametrize("model", ["odd", "five"])
@pytest.mark.parametrize("lens", [[(700, 1), (20, 2)], [(200, 50), (0, 33)], [(30, 1)] * 70])
def test_as_over_a_bf16_cache_of_the_same_values(model, lens):
    """The codes' values are bf16 numbers, and what follows the decoding is the same: equal outputs to the bit from the chunk kernel; the split kernel adds the
    products of a score in another order of the channels: both within their bounds"""
    st = Q.Step(*HEADS[model], lens, 32, seed=13).upload()
    out, lse = st.call(B.tkphi_quant_attention, st.config(workgroups=5))
    t = st.dev
    cfg = B.make_paged_config(st.hq, st.hkv, st.d, "bf16", st.d ** -0.5, t["K"], t["V"], workgroups=5)
    again, again_lse = P.Step.call(st, B.tkphi_paged_attention, cfg)
    if st.max_new >= 33:
        assert np.array_equal(out, again) and np.array_equal(lse, again_lse)
    else:
        want = P.attention_oracle(st)
        P.check(st, out, lse, want)
        P.check(st, again, again_lse, want)


def test_strided_rows_and_no_lse():
    st = Q.Step(14, 2, 64, [(50, 2), (20, 40)], 16).upload()
    wide = torch.full((st.rows, 18, 96), 7.0, device="cuda", dtype=torch.bfloat16)
    wide[:, 2:16, 8:72] = st.dev["q"]
    io_out = torch.full((st.rows, 16, 80), 7.0, device="cuda", dtype=torch.bfloat16)
    cfg, step = st.config(), st.step()
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    B.tkphi_quant_attention(cfg, step, st.pool(), B.make_attention_rows(wide[:, 2:16, 8:72], io_out[:, 1:15, 8:72]), ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    torch.cuda.synchronize()
    P.check(st, io_out[:, 1:15, 8:72].double().cpu().numpy(), None, P.attention_oracle(st))
    assert (io_out[:, 0] == 7).all() and (io_out[:, 15] == 7).all() and (io_out[:, :, :8] == 7).all() and (io_out[:, :, 72:] == 7).all()


def test_pool_beyond_32_bits():
    """Pages more than 2^32 bytes apart"""
    hq, hkv, d, page = 4, 2, 64, 16
    for lens in ([(90, 1), (60, 5)], [(90, 40), (10, 20)]):
        n_pages = (1 << 32) // (hkv * page * d) + 40
        st = Q.Step(hq, hkv, d, lens, page, seed=6)
        used = sorted(set(int(x) for x in st.table.reshape(-1) if x >= 0))
        place = {p: (n_pages - 1 - 3 * i if i % 2 else p) for i, p in enumerate(used)}
        big = {"K8": torch.zeros(n_pages, hkv, page, d, device="cuda", dtype=torch.uint8), "V8": torch.zeros(n_pages, hkv, page, d, device="cuda", dtype=torch.uint8),
               "S": torch.full((n_pages, hkv, page, 2), 127, device="cuda", dtype=torch.uint8)}
        for name, x in big.items():
            src = getattr(st, name).view(torch.uint8)
            for p, to in place.items():
                x[to] = src[p].cuda()
        want = P.attention_oracle(st)
        st.table = np.vectorize(lambda p: place.get(int(p), -1))(st.table).astype(np.int32)
        st.upload()
        st.dev.update(K8=big["K8"].view(torch.float8_e4m3fn), V8=big["V8"].view(torch.float8_e4m3fn), S=big["S"])
        out, lse = st.call(B.tkphi_quant_attention, st.config())
        P.check(st, out, lse, want)


@pytest.mark.parametrize("model", ["mha", "five"])
def test_long_pieces(model):
    """One workgroup passes over more tokens, and more pages, than it holds the page table of."""
    run(model, [(40000, 20)], 16, workgroups=1)
    run(model, [(40000, 20)], 16, workgroups=1, window=33000)
    run(model, [(5000, 20)], 1, workgroups=1)


# ---- blocks -----------------------------------------------------------------------------------------------------------------------
def blocks(heads, lens, page, block, first, last, top, workgroups=0, change=None, **kw):
    st = Q.Step(*heads, lens, page, block=block, **kw)
    if change:
        change(st)
    st.upload()
    out, lse = st.call(B.tkphi_quant_block_attention, st.config(first_blocks=first, last_blocks=last, top_blocks=top, workgroups=workgroups))
    P.check(st, out, None, P.block_oracle(st, first, last, top))
    assert (lse == 7.0).all()


@pytest.mark.parametrize("heads", [(32, 8, 64), (24, 8, 128), (1, 1, 64), (8, 1, 128), (14, 2, 64)])
@pytest.mark.parametrize("block,page,heads_first", [(16, 16, True), (32, 64, False), (64, 128, True)])
def test_blocks(heads, block, page, heads_first):
    blocks(heads, [(0, 1), (block - 1, 1), (block, 1), (9 * block - 1, 1), (9 * block, 1), (40 * block + 7, 1), (1500, 3)], page, block, 1, 2, 5, heads_first=heads_first)


@pytest.mark.parametrize("workgroups", [1, 2, 5, 64])
def test_blocks_with_work_cut_anywhere(workgroups):
    blocks((6, 2, 128), [(3000, 1), (17, 2)], 32, 32, 1, 2, 40, workgroups=workgroups)
    blocks((6, 2, 64), [(3000, 1), (17, 2)], 32, 32, 1, 2, 40, workgroups=workgroups)


def test_blocks_absent_pages_and_garbage():
    def gone(st):
        st.table[0, [2, 5]] = -1
        st.table[1, :] = -1
    blocks((4, 2, 64), [(400, 1), (90, 1)], 32, 16, 1, 2, 5, change=gone)
    blocks((4, 2, 128), [(333, 2), (18, 1)], 32, 16, 1, 1, 4, garbage=float("nan"))
    blocks((1, 1, 64), [(100, 700), (30, 2)], 16, 16, 1, 1, 4, slack_rows=3)


# ---- streams and graphs ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("lens", [[(3000, 1), (100, 1)], [(900, 70), (0, 20)]])
def test_repeats_bit_for_bit_also_from_a_graph_and_on_another_stream(lens):
    """A step of append, both attentions and a read back, on one workspace"""
    st = Q.Step(14, 2, 64, lens, 32, block=16).upload()
    t = st.dev
    gen = torch.Generator(device="cuda").manual_seed(3)
    qkv = torch.randn(st.rows, 18, 64, generator=gen, device="cuda").bfloat16()
    rows = torch.empty(4, st.rows, 14, 64, device="cuda", dtype=torch.bfloat16)
    back = torch.empty(2, st.rows, 2, 64, device="cuda", dtype=torch.bfloat16)
    freq = torch.from_numpy(500000.0 ** (-np.arange(0, 64, 2) / 64)).cuda()
    cfg, step, pool = st.config(rot_dim=64, first_blocks=1, last_blocks=2, top_blocks=20), st.step(), st.pool()
    size = B.tkphi_paged_workspace_bytes(cfg, step)
    ws = B.alloc_paged_workspace(size)
    new = B.make_new_rows(qkv[:, :14], qkv[:, 14:16], qkv[:, 16:], rows[0], inv_freq=freq)
    weight = torch.ones(64, device="cuda", dtype=torch.bfloat16)          # (structs hold addresses: the tensor stays here)
    norms = B.make_head_norms(weight, None, 1e-6)
    outputs = [rows, back, t["K8"].view(torch.uint8), t["V8"].view(torch.uint8), t["S"], t["M"], t["lse"]]

    def call():
        tail = (ws.data_ptr(), size, B.current_stream_ptr())
        B.tkphi_quant_append(cfg, step, pool, new, norms, *tail)
        B.tkphi_quant_attention(cfg, step, pool, B.make_attention_rows(rows[0], rows[1], t["lse"]), *tail)
        B.tkphi_quant_block_attention(cfg, step, pool, B.make_attention_rows(rows[0], rows[2]), *tail)
        B.tkphi_quant_read(cfg, step, pool, B.make_read_rows(back[0], back[1]), *tail)
    call()
    torch.cuda.synchronize()
    first = [x.clone() for x in outputs]

    def same():
        torch.cuda.synchronize()
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(outputs[:3], first[:3])) and all(torch.equal(x, y) for x, y in zip(outputs[3:], first[3:]))
        rows[1:3].fill_(7.0)
        back.fill_(7.0)
    rows[3] = 0
    first[0][3] = 0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        graph.replay()
        same()
        call()
        same()
    assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == 0
