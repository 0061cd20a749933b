"""tkphi_quant_attention over 64 channels with tokens outermost where two heads do not share an item: rows of codes are half lines, read with plain loads."""
import pytest

import paged_utils as P
import quant_utils as Q
from paper_2604_05438_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,lens", [((32, 8, 64), [(0, 3), (31, 3), (500, 3), (1500, 3), (62, 2)]), ((12, 3, 64), [(0, 1), (15, 1), (1500, 1)]), ((3, 3, 64), [(900, 20), (100, 5)]),
                                        ((14, 2, 64), [(400, 4), (7, 2)])])
@pytest.mark.parametrize("page,workgroups", [(16, 0), (8, 1), (104, 3), (100, 1), (64, 40)])
def test_heads_by_themselves_with_tokens_outermost(heads, lens, page, workgroups):
    """An odd number of heads, more query rows than two heads' share of a tile, or pages of no whole groups of 8 tokens"""
    for case in ("plain", "absent", "garbage", "window", "V"):
        window = 40 if case == "window" else 0
        st = Q.Step(*heads, lens, page, heads_first=False, seed=8, garbage=float("nan") if case == "garbage" else None, slack_rows=1)
        if case == "absent":
            st.table[-1, 0] = -1
        if case == "V":
            n = lens[-1][0]
            st.V8[st.table[-1, n // page], 1, n % page, 5] = float("nan")
            st.take_values()
        st.upload()
        out, lse = st.call(B.tkphi_quant_attention, st.config(window=window, workgroups=workgroups))
        P.check(st, out, lse, P.attention_oracle(st, window=window))
