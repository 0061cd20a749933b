"""A serving loop over one attention layer with a paged cache: prompts enter in chunks (append, attention of the chunk), then every
sequence decodes a token per step, first over everything cached, then over the blocks that score highest.  With --codes the cache is in 8 bits,
with --norms query and key heads are normed before they are rotated.

    python examples/paged_serving.py                     # 4 sequences of a 3B layer (24 / 8 heads of 128), prompts of 6000 tokens
    python examples/paged_serving.py --check             # small, every output against the float64 oracle
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_05438_amd.paged import PagedCache  # noqa: E402


def serve(hq=24, hkv=8, d=128, prompts=(6000, 4000, 5000, 3000), chunk=2048, steps=32, dtype="bf16", page=64, block=32, top=61, seed=0, on_step=None,
          codes=False, normed=False):
    """Returns the times in ms of (prompt chunks, dense steps, block steps).  on_step(cache, kind, new, qkv, out): called after every
    attention, before the step ends."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    total = [p + 2 * steps for p in prompts]
    n_pages = sum(-(-t // page) for t in total) + 4
    cache = PagedCache(hq, hkv, d, n_pages, page, len(prompts), max(chunk, len(prompts)), max(total), dtype, block=block, first_blocks=1, last_blocks=2,
                       top_blocks=top, codes=codes,
                       norms=(*(torch.rand(2, d, generator=gen, device="cuda") + 0.5).to(torch.bfloat16 if dtype == "bf16" else torch.float32), 1e-6) if normed else None)
    times = {"chunk": [], "dense": [], "blocks": []}

    def step(kind, new):
        cache.begin_step(new)
        rows = sum(new.values())
        qkv = torch.randn(rows, hq + 2 * hkv, d, generator=gen, device="cuda").to(cache.dtype)   # (the projections' output)
        q_rot, out = torch.empty(2, rows, hq, d, device="cuda", dtype=qkv.dtype)
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        cache.append(qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], q_rot)
        if kind == "blocks":
            cache.attend_blocks(q_rot, out)
        else:
            cache.attend(q_rot, out)
        b.record()
        times[kind].append((a, b))
        if on_step:
            on_step(cache, kind, new, qkv, out)
        cache.end_step()

    left = list(prompts)
    while any(left):                            # chunks of at most `chunk` tokens, of as many prompts as fit
        new, room = {}, chunk
        for i, n in enumerate(left):
            take = min(n, room)
            if take:
                new[i], left[i], room = take, n - take, room - take
        step("chunk", new)
    for kind in ("dense", "blocks"):
        for _ in range(steps):
            step(kind, {i: 1 for i in range(len(prompts))})
    torch.cuda.synchronize()
    assert cache.status() == 0
    return {k: [a.elapsed_time(b) for a, b in v] for k, v in times.items()}


def check(dtype="bf16", codes=False, normed=False):
    """A small run, every output against the oracle on the cache as it stands."""
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "tests"))
    import numpy as np
    import paged_utils as P
    from oracle import paged_oracle as O
    history = {}                                # sequence -> keys and values rotated by the oracle
    worst = [0.0]

    def on_step(cache, kind, new, qkv, out):
        hq, hkv, d = cache.cfg.n_q_heads, cache.cfg.n_kv_heads, cache.cfg.d_head
        x, y, freq = qkv.double().cpu().numpy(), out.double().cpu().numpy(), cache.inv_freq.cpu().numpy()
        K, V, M = (t.double().cpu().numpy() for t in (cache.K, cache.V, cache.M))
        half, row = P.HALF[dtype], 0
        keep = half
        if codes:                               # (an element is stored within half a step of its code, 2^-4 of it or 2^-10 of the row's power of two, at most 2^-8 of the largest)
            scales = cache.scales.double().cpu().numpy()
            K, V = K * np.exp2(scales[..., 0] - 127)[..., None], V * np.exp2(scales[..., 1] - 127)[..., None]
            keep = 2.0 ** -4
        qw, kw = (None if cache.norms is None else w.double().cpu().numpy() for w in (cache.norm_weights or (None, None)))
        for s, m in new.items():
            n = cache.length.get(s, 0)
            xq, xk = x[row:row + m, :hq], x[row:row + m, hq:hq + hkv]
            if normed:
                xq, xk = O.head_norm(xq, qw, 1e-6, 0.0), O.head_norm(xk, kw, 1e-6, 0.0)
            q = np.stack([O.rotate(xq[i], n + i, freq, False) for i in range(m)])
            q = torch.from_numpy(q).to(cache.dtype).double().numpy()
            k = np.stack([O.rotate(xk[i], n + i, freq, False) for i in range(m)])
            got, _ = O.gather(K, cache.pages[s], n + m)
            want = np.concatenate([history[s], k]) if s in history else k
            history[s] = want
            tiny = 2.0 ** -10 * np.abs(want).max(-1, keepdims=True) * 2.0 ** -7 if codes else 0.0
            assert (np.abs(np.swapaxes(got, 0, 1) - want) <= np.maximum(keep * np.abs(want) * 1.001, tiny) + 1e-5).all()
            c = cache.block_cfg
            ref = O.block_attention(q, K, V, M, cache.pages[s], n, m, c.score_scale, c.block, c.first_blocks, c.last_blocks, c.top_blocks) \
                if kind == "blocks" else O.paged_attention(q, K, V, cache.pages[s], n, m, c.score_scale)
            for i in range(m):
                for g in range(hq):
                    by, _ = P.bounds(dtype, d, n + m, *ref[i][g])
                    # (q is rotated and rounded here by the oracle, there by the kernel: where the two round apart, scores move by a step of q)
                    by = by + 2 * ref[i][g][2] * half * ref[i][g][3]
                    err = np.abs(y[row + i, g] - ref[i][g][0])
                    worst[0] = max(worst[0], float((err / by).max()))
                    assert (err <= by).all(), (kind, s, i, g)
            row += m
    serve(6, 2, 64, prompts=(150, 70, 33), chunk=96, steps=6, dtype=dtype, page=32, block=16, top=2, on_step=on_step, codes=codes,
          normed=normed)
    return worst[0]


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--check", action="store_true")
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--codes", action="store_true")
    ap.add_argument("--norms", action="store_true")
    args = ap.parse_args()
    if args.check:
        for dt in ("bf16", "f32"):
            print(f"{dt}: every output within its bound (at most {check(dt, args.codes and dt == 'bf16', args.norms):.2f} of it)")
    else:
        for kind, ms in serve(steps=args.steps, codes=args.codes, normed=args.norms).items():
            ms = sorted(ms)
            print(f"{kind}: {len(ms)} steps, median {ms[len(ms) // 2] * 1e3:.1f} us")
