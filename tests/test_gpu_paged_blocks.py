"""tkphi_block_attention against the float64 oracle: the blocks it sees, and the output over them."""
import numpy as np
import pytest
import torch

import paged_utils as P
from paper_2604_05438_amd import binding as B

pytestmark = pytest.mark.gpu


def run(dtype, heads, lens, page, block, first, last, top, seed=0, change=None, workgroups=0, **kw):
    hq, hkv, d = heads
    st = P.Step(dtype, hq, hkv, d, lens, page, block=block, seed=seed, **kw)
    if change:
        change(st)
    st.upload()
    out, lse = st.call(B.tkphi_block_attention, st.config(first_blocks=first, last_blocks=last, top_blocks=top, workgroups=workgroups))
    P.check(st, out, None, P.block_oracle(st, first, last, top))
    assert (lse == 7.0).all()
    return st


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [(32, 8, 64), (24, 8, 128), (1, 1, 64), (8, 1, 128), (14, 2, 64)])
@pytest.mark.parametrize("block,page", [(16, 16), (32, 64), (64, 128)])
def test_selection(dtype, heads, block, page):
    run(dtype, heads, [(0, 1), (block - 1, 1), (block, 1), (9 * block - 1, 1), (9 * block, 1), (40 * block + 7, 1), (1500, 3)], page, block, 1, 2, 5)


@pytest.mark.parametrize("first,last,top", [(0, 1, 0), (0, 1, 3), (3, 1, 0), (4, 4, 128), (0, 3, 1)])
def test_shares(first, last, top):
    run("bf16", (6, 2, 64), [(2000, 2), (100, 1), (700, 1)], 32, 16, first, last, top)


def test_long_lists_of_blocks():
    """More blocks than the selection takes at a step (1024), and several digits of the scores in common."""
    run("bf16", (2, 1, 64), [(40000, 2), (17000, 1)], 64, 16, 1, 2, 64)
    run("f32", (2, 1, 64), [(20000, 1)], 64, 16, 1, 2, 900)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_scores_go_to_the_lower_block(dtype):
    def same(st):
        st.M[:] = st.M[0, 0, 0]
    run(dtype, (2, 1, 64), [(5000, 1)], 64, 16, 1, 1, 20, change=same)

    def zero(st):                # scores of +0 and -0
        st.M[:] = 0
        st.M[::2] *= -1
    run(dtype, (2, 1, 64), [(5000, 1)], 64, 16, 1, 1, 20, change=zero)

    def few(st):                 # a handful of distinct rows
        st.M[:] = st.M[:3].repeat(st.n_pages // 3 + 1, 1, 1, 1)[:st.n_pages]
    run(dtype, (2, 1, 64), [(5000, 2)], 64, 16, 1, 1, 50, change=few)


def test_close_scores_are_told_apart():
    """fp32 means that differ in their last bits: sums in 32 bits would not order them."""
    def close(st):
        st.M[:] = st.M[0, 0, 0]
        r = torch.Generator().manual_seed(1)
        st.M *= 1 + torch.randint(-8, 9, st.M.shape, generator=r) * 2.0 ** -23
    run("f32", (2, 1, 64), [(9000, 1)], 64, 16, 0, 1, 100, change=close)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_means_that_are_no_numbers(bad):
    """NaN and -inf are not retrieved; +inf comes first."""
    def some(st):
        for b in (3, 9, 30, 31):
            st.M[st.table[0, b // 4], 0, b % 4, 7] = bad
        st.q[:, :, 7] = st.q[:, :, 7].abs() + 0.5
    run("bf16", (4, 1, 64), [(1000, 2)], 64, 16, 1, 1, 12, change=some)

    def every(st):
        st.M[:] = bad
        st.q[:] = st.q.abs() + 0.1
    run("bf16", (4, 1, 64), [(1000, 2)], 64, 16, 1, 1, 12, change=every)


def test_garbage_elsewhere_does_not_matter():
    run("bf16", (4, 2, 64), [(333, 2), (18, 1)], 32, 16, 1, 1, 4, garbage=float("nan"))
    run("f32", (4, 2, 64), [(333, 2), (18, 1)], 32, 16, 1, 1, 4, garbage=float("inf"), heads_first=False)


@pytest.mark.parametrize("workgroups", [1, 2, 5, 64])
def test_work_cut_anywhere(workgroups):
    run("bf16", (6, 2, 128), [(3000, 1), (17, 2)], 32, 32, 1, 2, 40, workgroups=workgroups)
    run("f32", (6, 2, 64), [(3000, 1), (17, 2)], 32, 32, 1, 2, 40, workgroups=workgroups)


def test_more_rows_than_the_workspace_holds_scores_for():
    run("bf16", (1, 1, 64), [(100, 700), (30, 2)], 16, 16, 1, 1, 4, slack_rows=3)


def test_absent_pages():
    def gone(st):
        st.table[0, [2, 5]] = -1
        st.table[1, :] = -1
    run("bf16", (4, 2, 64), [(400, 1), (90, 1)], 32, 16, 1, 2, 5, change=gone)


def test_same_in_a_graph():
    st = P.Step("bf16", 6, 2, 64, [(4000, 1), (900, 2)], 32, block=16).upload()
    cfg, step, t = st.config(first_blocks=1, last_blocks=2, top_blocks=30), st.step(), st.dev
    out, _ = st.call(B.tkphi_block_attention, cfg)
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    io, pool = B.make_attention_rows(t["q"], t["out"]), B.make_pool(t["K"], t["V"], t["M"])

    def call():
        B.tkphi_block_attention(cfg, step, pool, io, ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        t["out"].fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(t["out"].double().cpu().numpy(), out)
        call()
        torch.cuda.synchronize()
        assert np.array_equal(t["out"].double().cpu().numpy(), out)


def leave(st, keep):
    """No block's mean but those of `keep` (numbers of the first sequence) is a number."""
    per = st.page // st.block
    old = st.M.clone()
    st.M[:] = float("nan")
    for b in keep:
        st.M[st.table[0, b // per], :, b % per] = old[st.table[0, b // per], :, b % per]


@pytest.mark.parametrize("count", [0, 1, 11, 12, 13])
def test_about_as_many_candidates_as_are_retrieved(count):
    """Twelve are: fewer, exactly as many (the edge is the last of them), one more; in one step of the selection and in several."""
    r = np.random.default_rng(count)
    run("bf16", (4, 2, 64), [(5000, 1)], 64, 16, 1, 1, 12, change=lambda st: leave(st, r.choice(np.arange(2, 300), count, replace=False)))
    run("bf16", (2, 1, 64), [(135000, 1)], 64, 16, 1, 1, 12, change=lambda st: leave(st, r.choice(np.arange(2, 8400), count, replace=False)))


@pytest.mark.parametrize("tokens", [30000, 140000])
@pytest.mark.parametrize("kind", ["any", "same", "few", "close"])
def test_long_lists_and_full_bins(tokens, kind):
    """1875 blocks, which the threads hold, and 8750, which they do not; scores anywhere, and more than 1024 of them in one bin of the histogram."""
    def change(st):
        if kind == "same":
            st.M[:] = st.M[0, 0, 0]
        elif kind == "few":
            st.M[:] = st.M[:2].repeat(st.n_pages // 2 + 1, 1, 1, 1)[:st.n_pages]
        elif kind == "close":
            r = torch.Generator().manual_seed(2)
            st.M[:] = st.M[0, 0, 0] * (1 + torch.randint(-900, 900, st.M.shape, generator=r) * 2.0 ** -23)
    run("f32" if kind == "close" else "bf16", (2, 1, 64), [(tokens, 1)], 64, 16, 1, 2, 64, change=change, seed=9)
    run("f32", (1, 1, 64), [(tokens, 2)], 64, 16, 0, 1, 1000, change=change, seed=10)
