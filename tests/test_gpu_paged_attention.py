"""tkphi_paged_attention against the float64 oracle, element by element with bounds counted from the roundings (tests/paged_utils.py)."""
import numpy as np
import pytest
import torch

import paged_utils as P
from paper_2604_05438_amd import binding as B

pytestmark = pytest.mark.gpu

HEADS = {"1b": (32, 8, 64), "3b": (24, 8, 128), "one": (1, 1, 64), "wide": (8, 1, 128), "odd": (14, 2, 64), "five": (10, 2, 128), "mha": (3, 3, 64)}


def run(dtype, model, lens, page, window=0, workgroups=0, heads_first=True, seed=0, scale=None, **kw):
    hq, hkv, d = HEADS[model]
    st = P.Step(dtype, hq, hkv, d, lens, page, heads_first, seed=seed, **kw).upload()
    cfg = st.config(window=window, workgroups=workgroups, **({} if scale is None else {"scale": scale}))
    out, lse = st.call(B.tkphi_paged_attention, cfg)
    P.check(st, out, lse, P.attention_oracle(st, scale=scale, window=window))
    return st


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("model", ["one", "1b", "3b", "wide", "odd", "five", "mha"])
def test_single_tokens(dtype, model):
    """From a lone token to some hundreds, across tile and page ends."""
    run(dtype, model, [(0, 1), (1, 1), (14, 1), (15, 1), (16, 1), (31, 1), (127, 1), (128, 1), (500, 1)], 16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,heads_first", [(1, True), (7, False), (24, True), (64, False), (100, True), (256, False)])
def test_pages_and_orders(dtype, page, heads_first):
    run(dtype, "odd", [(77, 1), (0, 3), (300, 2), (255, 1)], page, heads_first=heads_first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("model", ["one", "3b", "wide", "odd"])
@pytest.mark.parametrize("lens", [[(40, 5)], [(0, 17), (33, 4), (100, 1)], [(0, 70), (61, 40), (5, 0), (200, 3)], [(130, 150)]])
def test_chunks(dtype, model, lens):
    run(dtype, model, lens, 16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 5, 64, 129])
@pytest.mark.parametrize("lens", [[(300, 1), (3, 1), (64, 1)], [(0, 90), (200, 33)]])
def test_windows(dtype, window, lens):
    run(dtype, "five", lens, 24, window=window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("workgroups", [1, 2, 3, 7, 40, 333])
def test_work_cut_anywhere(dtype, workgroups):
    """Items whole, shared by several workgroups, several items per workgroup; single tokens and chunks."""
    run(dtype, "odd", [(900, 1), (5, 1), (2000, 2), (0, 1)], 32, workgroups=workgroups)
    run(dtype, "odd", [(700, 40), (0, 90), (64, 1)], 32, workgroups=workgroups, seed=3)


def test_many_sequences():
    r = np.random.default_rng(5)
    run("bf16", "one", [(int(r.integers(0, 60)), int(r.integers(0, 3))) for _ in range(150)], 16, slack_rows=3)


def test_rows_in_another_order_than_the_sequences():
    run("f32", "odd", [(20, 2), (0, 3), (50, 1)], 16, order=[2, 0, 1], slack_rows=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("garbage", [float("nan"), float("inf"), float("-inf")])
def test_what_nobody_sees_may_hold_anything(dtype, garbage):
    """Rows of pages behind the end, pages of nobody, tokens behind every window."""
    run(dtype, "odd", [(37, 1), (0, 1), (150, 3)], 32, garbage=garbage)
    run(dtype, "odd", [(37, 40), (0, 33)], 100, garbage=garbage, window=20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("odd", [float("nan"), float("inf")])
def test_later_tokens_do_not_touch_earlier_queries(dtype, odd):
    """A value of token 60 that is no number, or infinite: the queries before it do not notice, those from it on do (NaN or
    infinity); the same for a key."""
    for lens, token, window in (([(50, 30)], 60, 0), ([(0, 120)], 60, 20), ([(58, 4)], 60, 0)):
        st = P.Step(dtype, 14, 2, 64, lens, 16, seed=8)
        for pool in (st.V, st.K):
            st2 = P.Step(dtype, 14, 2, 64, lens, 16, seed=8)
            x = st2.V if pool is st.V else st2.K
            x[st2.table[0, token // 16], 1, token % 16, 5] = odd
            st2.upload()
            out, lse = st2.call(B.tkphi_paged_attention, st2.config(window=window))
            want = P.attention_oracle(st2, window=window)
            n = lens[0][0]
            clean = [i for i in range(lens[0][1]) if n + i < token or (window and n + i >= token + window)]
            for i in clean:
                for g in range(14):
                    by, bl = P.bounds(dtype, 64, n + i, *want[0][i][g])
                    assert (np.abs(out[i, g] - want[0][i][g][0]) <= by).all() and abs(lse[i, g] - want[0][i][g][1]) <= bl, (i, g)
            assert len(clean) < lens[0][1]
            dirty = [i for i in range(lens[0][1]) if i not in clean]
            for i in dirty:
                for g in range(7):                   # the other KV head
                    by, _ = P.bounds(dtype, 64, n + i, *want[0][i][g])
                    assert (np.abs(out[i, g] - want[0][i][g][0]) <= by).all()
                if x is st2.V:
                    assert not np.isfinite(out[i, 7:, 5]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_absent_pages_are_seen_by_nobody(dtype):
    lens = [(100, 1), (40, 30), (30, 1), (3, 2)]
    st = P.Step(dtype, 14, 2, 64, lens, 16, seed=2)
    st.table[0, 2] = -1
    st.table[1, [0, 3]] = -1
    st.table[2, :] = -1               # nothing at all: 0 and -inf
    st.table[3, 0] = -1
    st.upload()
    out, lse = st.call(B.tkphi_paged_attention, st.config())
    P.check(st, out, lse, P.attention_oracle(st))
    assert (out[st.first[2]] == 0).all() and np.isneginf(lse[st.first[2]]).all()
    # a window whose every page is absent
    st = P.Step(dtype, 14, 2, 64, [(100, 1), (90, 20)], 16, seed=2)
    st.table[0, 5:] = -1
    st.table[1, :] = -1
    st.upload()
    out, lse = st.call(B.tkphi_paged_attention, st.config(window=10))
    P.check(st, out, lse, P.attention_oracle(st, window=10))


def test_bad_descriptions_are_skipped_and_reported():
    lens = [(20, 1), (30, 2), (10, 1), (5, 1), (6, 1)]
    for i, word, value in ((1, 0, -1), (1, 1, -2), (2, 0, 1000), (2, 2, 6), (3, 2, -1), (4, 1, 3)):
        st = P.Step("bf16", 14, 2, 64, lens, 16)
        st.seqs[i, word] = value
        st.upload()
        out, lse = st.call(B.tkphi_paged_attention, st.config(), check_status=B.TKPHI_DEV_BAD_LENGTH)
        P.check(st, out, lse, P.attention_oracle(st), skip=(i,))
    for value in (-2, 10 ** 9, 14):
        st = P.Step("bf16", 14, 2, 64, lens, 16)
        st.table[0, 1] = value if value != 14 else st.n_pages
        st.upload()
        out, lse = st.call(B.tkphi_paged_attention, st.config(), check_status=B.TKPHI_DEV_BAD_PAGE)
        P.check(st, out, lse, P.attention_oracle(st))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loud_scores(dtype):
    """Scores far apart: the running maximum moves by hundreds, weights underflow."""
    run(dtype, "five", [(400, 1), (100, 20)], 16, scale=12.0, seed=4)
    run(dtype, "five", [(400, 1), (100, 20)], 16, scale=1e-6, seed=4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_rows_and_no_lse(dtype):
    st = P.Step(dtype, 14, 2, 64, [(50, 2), (20, 40)], 16).upload()
    wide = torch.full((st.rows, 18, 96), 7.0, device="cuda", dtype=P.dt(dtype))
    wide[:, 2:16, 8:72] = st.dev["q"]
    st.dev["q"], st.dev["lse"] = wide[:, 2:16, 8:72], None
    io_out = torch.full((st.rows, 16, 80), 7.0, device="cuda", dtype=P.dt(dtype))
    t = st.dev
    cfg, step = st.config(), st.step()
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    B.tkphi_paged_attention(cfg, step, B.make_pool(t["K"], t["V"]), B.make_attention_rows(t["q"], io_out[:, 1:15, 8:72]), ws.data_ptr(), ws.numel(),
                            B.current_stream_ptr())
    torch.cuda.synchronize()
    P.check(st, io_out[:, 1:15, 8:72].double().cpu().numpy(), None, P.attention_oracle(st))
    assert (io_out[:, 0] == 7).all() and (io_out[:, 15] == 7).all() and (io_out[:, :, :8] == 7).all() and (io_out[:, :, 72:] == 7).all()


def test_repeats_bit_for_bit_also_from_a_graph_and_on_another_stream():
    for lens in ([(3000, 1), (100, 1)], [(900, 70), (0, 20)]):
        st = P.Step("bf16", 14, 2, 64, lens, 32).upload()
        cfg, step, t = st.config(), st.step(), st.dev
        out, lse = st.call(B.tkphi_paged_attention, cfg)
        ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
        io, pool = B.make_attention_rows(t["q"], t["out"], t["lse"]), B.make_pool(t["K"], t["V"])

        def call():
            B.tkphi_paged_attention(cfg, step, pool, io, ws.data_ptr(), ws.numel(), B.current_stream_ptr())
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            call()
        torch.cuda.synchronize()
        assert np.array_equal(t["out"].double().cpu().numpy(), out)
        with torch.cuda.graph(graph):
            call()
        for _ in range(4):
            t["out"].fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            assert np.array_equal(t["out"].double().cpu().numpy(), out) and np.array_equal(t["lse"].double().cpu().numpy(), lse)
            t["out"].fill_(7.0)
            call()
            torch.cuda.synchronize()
            assert np.array_equal(t["out"].double().cpu().numpy(), out)


def test_pool_beyond_32_bits():
    """Pages more than 2^32 bytes (and elements) apart."""
    hq, hkv, d, page = 4, 2, 64, 16
    n_pages = (1 << 32) // (hkv * page * d) + 40        # elements past 2^32: 8.6 GB of bf16
    K = torch.zeros(n_pages, hkv, page, d, device="cuda", dtype=torch.bfloat16)
    V = torch.zeros_like(K)
    st = P.Step("bf16", hq, hkv, d, [(90, 1), (60, 5)], page, seed=6)
    used = sorted(set(int(x) for x in st.table.reshape(-1) if x >= 0))
    for name, big in (("K", K), ("V", V)):
        for i, p in enumerate(used):
            big[n_pages - 1 - 3 * i if i % 2 else p] = getattr(st, name)[p].cuda()
    place = {p: (n_pages - 1 - 3 * i if i % 2 else p) for i, p in enumerate(used)}
    want = P.attention_oracle(st)
    st.table = np.vectorize(lambda p: place.get(int(p), -1))(st.table).astype(np.int32)
    st.upload()
    st.dev["K"], st.dev["V"] = K, V
    out, lse = st.call(B.tkphi_paged_attention, st.config())
    P.check(st, out, lse, want)


@pytest.mark.parametrize("model", ["mha", "five"])
def test_long_pieces(model):
    """One workgroup passes over more tokens, and more pages, than it holds the page table of."""
    run("bf16", model, [(40000, 20)], 16, workgroups=1)
    run("bf16", model, [(40000, 20)], 16, workgroups=1, window=33000)
    run("bf16", model, [(5000, 20)], 1, workgroups=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_sequences_of_several_tokens(dtype):
    r = np.random.default_rng(6)
    run(dtype, "five", [(int(r.integers(0, 90)), int(r.integers(0, 12))) for _ in range(90)], 16, slack_rows=1)
    run(dtype, "wide", [(int(r.integers(0, 90)), int(r.integers(0, 2))) for _ in range(90)], 16, workgroups=50)


def test_sequences_that_share_rows_do_no_harm():
    """More items than the rows allow for: what fits is done, the rest is left out and reported; memory stays whole."""
    st = P.Step("bf16", 14, 2, 64, [(0, 40)] * 30, 16, seed=1)
    st.seqs[:, 2] = 0
    st.rows, st.q = 40, st.q[:40]
    st.upload()
    out, lse = st.call(B.tkphi_paged_attention, st.config(), check_status=B.TKPHI_DEV_BAD_LENGTH)
    assert np.isfinite(out).all()


@pytest.mark.parametrize("model", ["odd", "five"])
@pytest.mark.parametrize("lens,workgroups", [([(1000, 64), (5, 40)], 0), ([(1000, 64), (5, 40)], 1), ([(3000, 1), (70, 2)], 0), ([(3000, 1), (70, 2)], 1)])
@pytest.mark.parametrize("scale", [1.0, 0.125, 0.02])
def test_a_mean_of_equal_values_is_that_value(model, lens, workgroups, scale):
    """Where all values are 1 the output is 1 whatever the weights: what their rounding takes from the product it takes from the divisor.  Sums in
    32 bits are off by far less than the 2^-9 at which the output would round to the number below 1."""
    hq, hkv, d = HEADS[model]
    st = P.Step("bf16", hq, hkv, d, lens, 16, seed=11)
    st.V[:] = 1.0
    st.upload()
    out, lse = st.call(B.tkphi_paged_attention, st.config(scale=scale, workgroups=workgroups))
    P.check(st, out, lse, P.attention_oracle(st, scale=scale))
    assert (out == 1.0).all(), (out != 1.0).mean()


@pytest.mark.parametrize("model", ["odd", "five"])
@pytest.mark.parametrize("fresh", [1, 40])
def test_equal_weights_below_a_peak(model, fresh):
    """One token with the highest score and many with the same lower one, whose weight lies between two numbers of 8 bits: every one of them is rounded
    the same way."""
    hq, hkv, d = HEADS[model]
    for lag in (0.3, 0.51, 5.3, -float(np.log2(0.5 + 0.9 * 2.0 ** -9)), -float(np.log2(0.5 + 1.1 * 2.0 ** -9))):      # (0.9: half a step down, all but)
        st = P.Step("bf16", hq, hkv, d, [(300, fresh)], 16, seed=12)
        st.K[:] = 0
        st.K[..., 0] = 4.0
        st.K[st.table[0, 12], :, 5, 0] = 6.0              # token 197
        st.q[:] = 0
        st.q[..., 0] = 1.0
        st.V[:] = 1.0
        scale = lag * 0.6931471805599453 / 2              # exponents of 2 between the two scores
        st.upload()
        out, lse = st.call(B.tkphi_paged_attention, st.config(scale=scale))
        P.check(st, out, lse, P.attention_oracle(st, scale=scale))
        assert (out == 1.0).all(), (lag, (out != 1.0).mean())


def test_more_items_than_32_bits_of_sequences_that_share_rows():
    """1024 sequences of 2^23 new tokens on the same rows, 2^31 items among them, and some of one token behind them: what fits is done, the rest is
    left out and reported.  No page is there, so all outputs are 0 (rows and heads of q and of out overlap in memory, to be small)."""
    n, rows, hq, d = 1100, 1 << 23, 8, 64
    seqs = torch.zeros(n, 4, dtype=torch.int32)
    seqs[:1024, 1] = rows
    seqs[1024:, 1] = 1
    seqs, pages = seqs.cuda(), torch.full((n, 1), -1, dtype=torch.int32, device="cuda")
    K = torch.zeros(2, 1, 16, d, device="cuda")
    q = torch.ones((rows + hq - 1) * d, device="cuda").as_strided((rows, hq, d), (d, d, 1))
    flat = torch.full(((rows + hq - 1) * d,), 7.0, device="cuda")
    out = flat.as_strided((rows, hq, d), (d, d, 1))
    cfg = B.make_paged_config(hq, 1, d, "f32", 0.125, K, K, window=1)
    step = B.make_step(seqs, pages, rows, rows, rows)
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    assert ws.numel() > 256, B.tkphi_last_error()
    B.tkphi_paged_attention(cfg, step, B.make_pool(K, K), B.make_attention_rows(q, out), ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == B.TKPHI_DEV_BAD_LENGTH
    assert (flat == 0).all()
