"""Paged-cache steps for the tests: random pools, page tables and sequences on the CPU and the device, and the bounds on what the kernels
may be off, counted from their roundings (half a step of a type is finfo(t).eps / 2: bf16 2^-8, fp32 2^-24)."""
from __future__ import annotations

import numpy as np
import torch

from oracle import paged_oracle as O
from paper_2604_05438_amd import binding as B

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U = 2.0 ** -24


def dt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


class Step:
    """A step of `lens` = [(cached, new)] sequences.  Pages lie in random order; tail: entries of the table behind the end."""

    def __init__(self, dtype, hq, hkv, d, lens, page, heads_first=True, block=0, seed=0, slack_rows=0, device="cuda", garbage=None, order=None):
        r = np.random.default_rng(seed)
        self.dtype, self.hq, self.hkv, self.d, self.lens, self.page, self.block, self.device = dtype, hq, hkv, d, lens, page, block, device
        count = [-(-(n + m) // page) for n, m in lens]
        self.n_pages = sum(count) + 2
        ids = r.permutation(self.n_pages)
        self.table = np.full((len(lens), max(count + [1])), -1, dtype=np.int32)
        at = 0
        for i, c in enumerate(count):
            self.table[i, :c] = ids[at:at + c]
            at += c
        self.first, row = [0] * len(lens), 0
        for i in (order if order is not None else range(len(lens))):
            self.first[i] = row
            row += lens[i][1]
        self.rows = row + slack_rows
        self.seqs = np.array([[n, m, f, 0] for (n, m), f in zip(lens, self.first)], dtype=np.int32).reshape(-1, 4)
        self.max_new, self.max_len = max([m for _, m in lens] + [0]), max([n + m for n, m in lens] + [0])
        gen = torch.Generator().manual_seed(seed + 1)
        shape = (self.n_pages, hkv, page, d) if heads_first else (self.n_pages, page, hkv, d)

        def pool():
            x = torch.randn(shape, generator=gen).to(dt(dtype))
            x = x if heads_first else x.transpose(1, 2)
            if garbage is not None:           # whatever no sequence owns
                own = torch.zeros(self.n_pages, page, dtype=torch.bool)
                for i, (n, m) in enumerate(lens):
                    for t in range(n + m):
                        own[self.table[i, t // page], t % page] = True
                x.transpose(1, 2)[~own] = garbage
            return x

        self.K, self.V = pool(), pool()
        self.q = (torch.randn(self.rows, hq, d, generator=gen) * 1.5).to(dt(dtype))
        self.M = None
        if block:
            self.M = torch.nan_to_num(self.K.float()).unflatten(2, (page // block, block)).mean(3).to(dt(dtype)).contiguous()

    def upload(self):
        """On the device, in the same memory order (strides included)."""
        def up(x):
            if x is None:
                return None
            if x.is_contiguous():
                return x.to(self.device)
            return x.transpose(1, 2).contiguous().to(self.device).transpose(1, 2)
        self.dev = {n: up(getattr(self, n)) for n in ("K", "V", "M", "q")}
        self.dev["seqs"] = torch.from_numpy(self.seqs).to(self.device)
        self.dev["pages"] = torch.from_numpy(self.table).to(self.device)
        self.dev["out"] = torch.full((self.rows, self.hq, self.d), 7.0, device=self.device, dtype=dt(self.dtype))
        self.dev["lse"] = torch.full((self.rows, self.hq), 7.0, device=self.device)
        return self

    def config(self, **kw):
        return B.make_paged_config(self.hq, self.hkv, self.d, self.dtype, kw.pop("scale", self.d ** -0.5), self.K, self.V, block=self.block, **kw)

    def step(self):
        t = self.dev
        return B.make_step(t["seqs"], t["pages"], self.rows, self.max_new, self.max_len)

    def call(self, fn, cfg, ws=None, check_status=0):
        """fn over out and lse; returns them on the CPU as float64"""
        t = self.dev
        io = B.make_attention_rows(t["q"], t["out"], t["lse"])
        size = B.tkphi_paged_workspace_bytes(cfg, self.step())
        assert size > 0, B.tkphi_last_error()
        ws = B.alloc_paged_workspace(size) if ws is None else ws
        fn(cfg, self.step(), B.make_pool(t["K"], t["V"], t["M"]), io, ws.data_ptr(), ws.numel(), B.current_stream_ptr())
        assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == check_status
        assert (ws[256:256 + 4096] == 0).all()          # the counters are left at zero
        return t["out"].double().cpu().numpy(), t["lse"].double().cpu().numpy()


def f64(x):
    return x.double().numpy()


def bounds(dtype, d, tokens, y, lse, spread, reach):
    """What out and lse may be off.  A score is a sum of d products in 32 bits (each addition rounds by U of at most `reach`, the sum of
    the products' sizes), scaled and exponentiated in base 2 (a handful of roundings of values up to reach): dx.  That changes every
    weight by a factor of at most e^(2 dx) against the sum; sums over tokens run in chains of at most tokens / 64 terms per lane with one rescaling
    each, joined over lanes, wavefronts and pieces (64 more).  bf16: every weight is rounded for the product with V (half a step),
    and so is the output."""
    dx = U * ((d + 8) * reach + 8)
    chain = U * (2 * tokens / 16 + 128)
    rel = np.expm1(2 * dx) + chain + (HALF["bf16"] if dtype == "bf16" else 0.0)
    return (rel * spread * (1 + HALF[dtype]) + HALF[dtype] * np.abs(y)) * (1 + 2.0 ** -20) + 1e-37, dx + chain + 4 * U * (abs(lse) + 1)


def check(st: Step, out, lse, want, skip=()):
    """want: per sequence the oracle's results; rows of no sequence and of the sequences in `skip` are untouched"""
    touched = np.zeros(st.rows, dtype=bool)
    for i, (n, m) in enumerate(st.lens):
        if i in skip:
            continue
        for k in range(m):
            row = st.first[i] + k
            touched[row] = True
            for g in range(st.hq):
                y, l, spread, reach = want[i][k][g]
                by, bl = bounds(st.dtype, st.d, n + m, y, l, spread, reach)
                got = out[row, g]
                finite = np.isfinite(y)
                assert np.isnan(got[~finite]).all() or np.array_equal(got[~finite], y[~finite]), (i, k, g)
                err = np.abs(got - y)[finite]
                assert (err <= by[finite]).all(), (i, k, g, float(np.nanmax(err / by[finite])))
                if lse is not None:
                    if np.isfinite(l):
                        assert abs(lse[row, g] - l) <= bl, (i, k, g, lse[row, g], l, bl)
                    else:
                        assert lse[row, g] == l or np.isnan(l), (i, k, g, lse[row, g], l)
    assert (out[~touched] == 7.0).all()
    if lse is not None:
        assert (lse[~touched] == 7.0).all()


def attention_oracle(st: Step, scale=None, window=0, table=None):
    table = st.table if table is None else table
    K, V, q = f64(st.K), f64(st.V), f64(st.q)
    scale = float(np.float32(st.d ** -0.5 if scale is None else scale))
    return [O.paged_attention(q[f:f + m], K, V, table[i], n, m, scale, window) for i, ((n, m), f) in enumerate(zip(st.lens, st.first))]


def block_oracle(st: Step, first, last, top, scale=None):
    K, V, q, M = f64(st.K), f64(st.V), f64(st.q), f64(st.M)
    scale = float(np.float32(st.d ** -0.5 if scale is None else scale))
    return [O.block_attention(q[f:f + m], K, V, M, st.table[i], n, m, scale, st.block, first, last, top)
            for i, ((n, m), f) in enumerate(zip(st.lens, st.first))]
