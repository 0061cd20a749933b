"""Steps on a paged cache in 8 bits for the tests: a paged_utils.Step whose pool is quantised by the oracle, K and V being what the codes stand for (bf16
numbers), so that the oracle and the bounds of a bf16 cache hold."""
from __future__ import annotations

import numpy as np
import torch

import paged_utils as P
from oracle import paged_oracle as O
from paper_2604_05438_amd import binding as B


def quantise(x):
    """A tensor's rows -> codes in its memory order, exponent bytes"""
    codes, b = O.quantise(P.f64(x))
    codes = torch.from_numpy(codes).to(torch.float8_e4m3fn)
    if not x.is_contiguous():
        codes = codes.transpose(1, 2).contiguous().transpose(1, 2)
    return codes, torch.from_numpy(b).to(torch.uint8)


def values(codes, b):
    """What codes and bytes stand for, as bf16 in the codes' memory order (exact)"""
    return (codes.double() * torch.exp2(b.double() - 127)[..., None]).to(torch.bfloat16)


class Step(P.Step):
    def __init__(self, hq, hkv, d, lens, page, heads_first=True, change=None, **kw):
        super().__init__("bf16", hq, hkv, d, lens, page, heads_first, **kw)
        if change:
            change(self)
        self.requantise()

    def requantise(self):
        (self.K8, kb), (self.V8, vb) = quantise(self.K), quantise(self.V)
        self.S = torch.stack([kb, vb], -1).contiguous()
        self.take_values()

    def take_values(self):
        self.K, self.V = values(self.K8, self.S[..., 0]), values(self.V8, self.S[..., 1])

    def upload(self):
        super().upload()

        def up(x):
            return x.cuda() if x.is_contiguous() else x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        self.dev.update(K8=up(self.K8), V8=up(self.V8), S=self.S.cuda())
        return self

    def config(self, **kw):
        return B.make_paged_config(self.hq, self.hkv, self.d, "bf16", kw.pop("scale", self.d ** -0.5), self.K8, self.V8, block=self.block, **kw)

    def pool(self):
        return B.make_quant_pool(self.dev["K8"], self.dev["V8"], self.dev["S"], self.dev["M"])

    def call(self, fn, cfg, ws=None, check_status=0):
        t = self.dev
        io = B.make_attention_rows(t["q"], t["out"], t["lse"])
        size = B.tkphi_paged_workspace_bytes(cfg, self.step())
        assert size > 0, B.tkphi_last_error()
        ws = B.alloc_paged_workspace(size) if ws is None else ws
        fn(cfg, self.step(), self.pool(), io, ws.data_ptr(), ws.numel(), B.current_stream_ptr())
        assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == check_status
        assert (ws[256:256 + 4096] == 0).all()          # the counters are left at zero
        return t["out"].double().cpu().numpy(), None if t["lse"] is None else t["lse"].double().cpu().numpy()
