"""The serving example: prompts in chunks, dense steps, block steps on one cache, every output against the oracle; and the cache's bookkeeping."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_serving_loop(dtype):
    import paged_serving
    assert paged_serving.check(dtype) <= 1.0


def test_pages_are_taken_and_given_back():
    from paper_2604_05438_amd.paged import PagedCache
    c = PagedCache(4, 2, 64, 5, 16, 3, 40, 64, block=16, last_blocks=1, device="cpu")
    st = c.begin_step({"a": 17, "b": 3})
    assert (st.n_seqs, st.rows, st.max_new, st.max_len, st.max_pages) == (2, 20, 17, 17, 2)
    assert c._seqs.tolist() == [[0, 17, 0, 0], [0, 3, 17, 0]] and c._table.tolist() == [[0, 1], [2, -1]]
    c.end_step()
    c.begin_step({"b": 1, "a": 1})
    assert c._seqs.tolist() == [[3, 1, 0, 0], [17, 1, 1, 0]] and len(c.free) == 2
    c.end_step()
    with pytest.raises(MemoryError):
        c.begin_step({"a": 31, "d": 9})
    with pytest.raises(ValueError):
        c.begin_step({"a": 3, "d": 38})
    c.release("a")
    assert sorted(c.free) == [0, 1, 3, 4] and "a" not in c.length
    c.begin_step({"c": 40})
    assert len(c.pages["c"]) == 3


def test_sequences_released_within_a_step_are_gone():
    from paper_2604_05438_amd.paged import PagedCache
    c = PagedCache(4, 2, 64, 5, 16, 3, 40, 64, block=16, last_blocks=1, device="cpu")
    c.begin_step({"a": 17, "b": 3})
    c.release("a")
    c.end_step()
    assert c.length == {"b": 3} and set(c.pages) == {"b"} and len(c.free) == 4
    c.end_step()                          # (nothing to end)
    assert c.length == {"b": 3}
    c.begin_step({"a": 2, "b": 1})
    assert c._seqs.tolist() == [[0, 2, 0, 0], [3, 1, 2, 0]]
    c.end_step()
    c.release("a")
    c.end_step()
    assert c.length == {"b": 4} and len(c.free) == 4


def test_negative_numbers_of_tokens_are_refused():
    from paper_2604_05438_amd.paged import PagedCache
    c = PagedCache(4, 2, 64, 5, 16, 3, 40, 64, device="cpu")
    with pytest.raises(ValueError):
        c.begin_step({"a": 17, "b": -3})
    assert not c.pages and len(c.free) == 5
    c.begin_step({"a": 17, "b": 0})
    assert c._seqs.tolist() == [[0, 17, 0, 0], [0, 0, 17, 0]]


@pytest.mark.gpu
def test_calls_on_another_stream_keep_the_tables_of_their_step():
    """attend waits on a side stream while later steps begin on the default one: their tables must not take the memory of its own."""
    import torch
    from paper_2604_05438_amd.paged import PagedCache
    gen = torch.Generator(device="cuda").manual_seed(3)
    c = PagedCache(4, 2, 64, 12, 16, 4, 64, 96, dtype="f32")

    def rows(n, heads):
        return torch.randn(n, heads, 64, generator=gen, device="cuda")
    c.begin_step({"a": 50})
    out, q = torch.zeros(2, 50, 4, 64, device="cuda")
    c.append(rows(50, 4), rows(50, 2), rows(50, 2), q)
    c.end_step()
    c.begin_step({"a": 1})
    one, want, got = torch.zeros(3, 1, 4, 64, device="cuda")
    c.append(rows(1, 4), rows(1, 2), rows(1, 2), one)
    c.attend(one, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        c.attend(one, got)
    c.end_step()
    for s in ("b", "c", "d"):
        c.begin_step({s: 1})
        c.end_step()
    assert not side.query()
    torch.cuda.synchronize()
    assert c.status() == 0 and torch.equal(got, want) and not torch.equal(want, torch.zeros_like(want))
