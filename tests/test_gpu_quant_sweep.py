"""Seeded random steps of the calls on the cache in 8 bits and on normed heads: heads, pages, orders, lengths, windows, cuts of the work, absent pages, garbage."""
import random

import pytest

import paged_utils as P
import quant_utils as Q
import test_gpu_quant_append as A
from paper_2604_05438_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", range(8))
def test_random_steps(seed):
    r = random.Random(seed)
    for case in range(12):
        hkv, G, d = r.choice([1, 2, 2, 3, 4, 8]), r.choice([1, 1, 2, 3, 4, 5, 7, 8]), r.choice([64, 64, 128])
        page = r.choice([1, 3, 8, 16, 16, 24, 32, 48, 64, 100, 128])
        block = r.choice([0] + [b for b in (16, 32, 64) if page % b == 0])
        kind = r.choice(["single", "few", "chunk", "mixed", "many"])
        lens = []
        for _ in range(r.randint(65, 80) if kind == "many" else r.randint(1, 6)):
            cached = r.choice([0, r.randint(0, 40), r.randint(0, 700), r.randint(0, 60 if kind == "many" else 2500)])
            lens.append((cached, {"single": 1, "few": r.randint(0, 8), "chunk": r.randint(1, 150), "mixed": r.choice([0, 1, 1, 2, 60]), "many": r.randint(0, 2)}[kind]))
        lens.append((r.randint(0, 90), 1))
        heads_first, garbage = r.random() < 0.5, r.choice([None, None, float("nan")])
        window, workgroups = r.choice([0, 0, 0, r.randint(1, 300)]), r.choice([0, 0, 0, 1, 2, 5, 17, 100])
        what = r.choice(["attend", "attend", "append", "read", "norm"] + (["blocks"] if block else []))
        print(seed, case, what, hkv, G, d, page, block, lens[:8], heads_first, window, workgroups, flush=True)
        if what == "norm":
            st = P.Step(r.choice(["bf16", "f32"]), hkv * G, hkv, d, lens, page, heads_first, block=block, seed=seed)
            A.check(st, r.choice([0, 16, d // 2, d]), r.random() < 0.5, r.choice(["shared", "heads", "ones"]), r.choice([0.0, 1.0]), with_q=r.random() < 0.8)
            continue
        st = Q.Step(hkv * G, hkv, d, lens, page, heads_first, block=block, seed=seed, garbage=garbage, slack_rows=r.randint(0, 2))
        if r.random() < 0.2:
            st.table[r.randrange(len(lens)), r.randrange(st.table.shape[1])] = -1
        lost = any(st.table[i, (n + j) // page] < 0 for i, (n, m) in enumerate(lens) for j in range(m))
        if what == "attend":
            st.upload()
            out, lse = st.call(B.tkphi_quant_attention, st.config(window=window, workgroups=workgroups))
            P.check(st, out, lse, P.attention_oracle(st, window=window))
        elif what == "blocks":
            first, last, top = r.randint(0, 3), r.randint(1, 3), r.randint(0, 20)
            st.upload()
            out, _ = st.call(B.tkphi_quant_block_attention, st.config(first_blocks=first, last_blocks=last, top_blocks=top, workgroups=min(workgroups, 64)))
            P.check(st, out, None, P.block_oracle(st, first, last, top))
        elif what == "append":
            A.check(st, r.choice([0, 16, d // 2, d]), r.random() < 0.5, r.choice([None, "shared", "heads", "ones"]), r.choice([0.0, 1.0]), with_q=r.random() < 0.8,
                    status=B.TKPHI_DEV_BAD_PAGE if lost else 0)
        else:
            A.read(st, status=B.TKPHI_DEV_BAD_PAGE if lost else 0, layout=r.choice(["rows", "heads"]))
