"""One workspace for many steps on the paged cache: large and small ones, with and without a plan, over blocks, with the work cut by hand.  Every output against
the float64 oracle, and the counters (the 4096 bytes from 256 on) at zero after every call."""
import pytest
import torch

import paged_utils as P
from paper_2604_05438_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_workspace_for_steps_of_all_sizes(dtype):
    hq, hkv, d, page, block = 8, 8, 64, 32, 16
    kept = dict(first_blocks=1, last_blocks=1, top_blocks=6)

    def step(lens, seed):
        return P.Step(dtype, hq, hkv, d, lens, page, block=block, seed=seed).upload()
    steps = {"chunk": step([(60, 100)], 1), "rows": step([(250, 200)], 2), "large": step([(20, 300), (100, 212)], 3),
             "tokens": step([(700, 1), (3, 1), (90, 1)], 4)}
    size = max(B.tkphi_paged_workspace_bytes(s.config(workgroups=w, **kept), s.step()) for s in steps.values() for w in (0, 4, 64))
    ws = B.alloc_paged_workspace(size)
    dense = {k: P.attention_oracle(s) for k, s in steps.items()}
    sparse = {k: P.block_oracle(s, 1, 1, 6) for k, s in steps.items()}
    for name, blocks, workgroups in [("chunk", False, 0), ("rows", True, 4), ("chunk", False, 64), ("large", True, 4), ("large", False, 0), ("rows", True, 0),
                                     ("tokens", False, 0), ("rows", True, 64), ("tokens", True, 0), ("large", False, 4), ("rows", True, 3), ("tokens", True, 64),
                                     ("tokens", False, 4), ("large", True, 0)]:
        s = steps[name]
        s.dev["out"].fill_(7.0)
        s.dev["lse"].fill_(7.0)
        cfg = s.config(workgroups=workgroups, **kept)
        out, lse = s.call(B.tkphi_block_attention if blocks else B.tkphi_paged_attention, cfg, ws=ws)
        P.check(s, out, None if blocks else lse, sparse[name] if blocks else dense[name])
    torch.cuda.synchronize()
