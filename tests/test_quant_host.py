"""The calls on the cache in 8 bits and on normed heads refuse what the host can see to be wrong before any launch; their oracle on small cases; PagedCache."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2604_05438_amd import binding as B
from paper_2604_05438_amd.paged import PagedCache


def good(**kw):
    cfg = B.tkphi_paged_config(32, 8, 64, B.TKPHI_BF16, 0.125, 32, 8 * 32 * 64, 32 * 64, 64, 0, 64, 0, 16, 1, 2, 8, 0)
    step = B.tkphi_step(4096, 4096, 3, 10, 20, 12, 300, 0)
    pool = B.tkphi_kv_pool(4096, 8192, 16384, 40, 0)
    codes = B.tkphi_quant_pool(4096, 8192, 12288, 16384, 40, 0)
    new = B.tkphi_new_rows(4096, 4096, 4096, 4096, 4096, 2048, 64, 512, 64, 512, 64, 2048, 64)
    att = B.tkphi_attention_rows(4096, 8192, 4096, 2048, 64, 2048, 64)
    read = B.tkphi_read_rows(4096, 8192, 512, 64, 512, 64)
    norms = B.tkphi_head_norms(4096, 8192, 64, 0, 1e-6, 1.0)
    got = {"cfg": cfg, "step": step, "pool": pool, "codes": codes, "new": new, "att": att, "read": read, "norms": norms}
    for name, value in kw.items():
        where, field = name.split("__")
        setattr(got[where], field, value)
    return got


CALLS = {"tkphi_norm_append": ("pool", "new", "norms"), "tkphi_quant_append": ("codes", "new", "norms"), "tkphi_quant_attention": ("codes", "att"),
         "tkphi_quant_block_attention": ("codes", "att"), "tkphi_quant_read": ("codes", "read")}


def status(call, ws=4096, short=0, none=(), **kw):
    g = good(**kw)
    size = B.tkphi_paged_workspace_bytes(good()["cfg"], good()["step"])
    args = [None if n in none else g[n] for n in ("cfg", "step", *CALLS[call])]
    return getattr(B.lib(), call)(*args, ws, size - short, None)


EVERY = [
    ("EINVAL", dict(cfg__kv_dtype=2)), ("ESHAPE", dict(cfg__n_q_heads=30)), ("ESHAPE", dict(cfg__d_head=96)), ("EINVAL", dict(cfg__score_scale=0.0)),
    ("ESHAPE", dict(cfg__page_tokens=0)), ("EALIGN", dict(cfg__stride_tok=60)), ("EALIGN", dict(cfg__stride_head=-64)), ("EALIGN", dict(cfg__stride_page=4)),
    ("EINVAL", dict(cfg__window=-1)), ("ESHAPE", dict(cfg__rot_dim=24)), ("ESHAPE", dict(cfg__block=8)), ("EINVAL", dict(step__n_seqs=-1)),
    ("EINVAL", dict(step__reserved=1)), ("EINVAL", dict(step__seqs=0)), ("EALIGN", dict(step__seqs=4100)), ("EINVAL", dict(step__pages=0)),
    ("EINVAL", dict(step__max_pages=0)), ("EALIGN", dict(step__pages=4098)),
]
POOL = [("EINVAL", "K", 0), ("EALIGN", "V", 8200), ("EINVAL", "n_pages", 0), ("EINVAL", "n_pages", -3), ("EINVAL", "reserved", 1)]


@pytest.mark.parametrize("call", CALLS)
def test_refusals_of_every_call(call):
    for want, kw in EVERY:
        assert status(call, **kw) == getattr(B, "TKPHI_" + want), (kw, B.tkphi_last_error())
        assert B.tkphi_last_error() != ""
    pool = CALLS[call][0]
    for want, field, value in POOL + ([("EINVAL", "scales", 0), ("EALIGN", "scales", 12290)] if pool == "codes" else []):
        assert status(call, **{f"{pool}__{field}": value}) == getattr(B, "TKPHI_" + want), (field, B.tkphi_last_error())
    if pool == "codes":       # bf16 rows only; strides are bytes there
        assert status(call, cfg__kv_dtype=B.TKPHI_F32) == B.TKPHI_EUNSUPPORTED
        for field in ("stride_tok", "stride_head", "stride_page"):
            assert status(call, **{f"cfg__{field}": 8 * 32 * 64 + 8}) == B.TKPHI_EALIGN
    assert status(call, ws=None) == B.TKPHI_EWORKSPACE and status(call, ws=4100) == B.TKPHI_EWORKSPACE and status(call, short=256) == B.TKPHI_EWORKSPACE
    for name in ("cfg", "step", *CALLS[call][:2]):
        assert status(call, none=(name,)) == B.TKPHI_EINVAL
    for kw in (dict(step__n_seqs=0, step__seqs=0), dict(step__rows=0), dict(step__max_new=0), dict(step__max_len=0)):
        assert status(call, **{f"{pool}__n_pages": 0}, **kw) == B.TKPHI_OK


@pytest.mark.parametrize("call", ["tkphi_norm_append", "tkphi_quant_append"])
def test_refusals_of_norms_and_rows(call):
    pool = CALLS[call][0]
    for want, kw in [
        ("EINVAL", dict(new__k=0)), ("EALIGN", dict(new__v=4104)), ("EINVAL", dict(new__q=0)), ("EINVAL", dict(new__q_rot=0)), ("EALIGN", dict(new__k_row=60)),
        ("EINVAL", dict(new__inv_freq=0)), ("EINVAL", {f"{pool}__M": 0}), ("EALIGN", {f"{pool}__M": 16392}),
        ("EINVAL", dict(norms__eps=0.0)), ("EINVAL", dict(norms__eps=-1e-6)), ("EINVAL", dict(norms__eps=float("nan"))), ("EINVAL", dict(norms__eps=float("inf"))),
        ("EINVAL", dict(norms__eps=1e-40)), ("EINVAL", dict(norms__weight_offset=float("nan"))), ("EINVAL", dict(norms__weight_offset=float("inf"))),
        ("EALIGN", dict(norms__q_weight=4104)), ("EALIGN", dict(norms__k_weight=4104)), ("EALIGN", dict(norms__q_weight_head=-64)),
        ("EALIGN", dict(norms__q_weight_head=63)), ("EALIGN", dict(norms__k_weight_head=32)),
    ]:
        assert status(call, **kw) == getattr(B, "TKPHI_" + want), (kw, B.tkphi_last_error())
    if call == "tkphi_norm_append":
        assert status(call, none=("norms",)) == B.TKPHI_EINVAL


def test_refusals_of_the_others():
    for want, call, kw in [
        ("EINVAL", "tkphi_quant_attention", dict(att__q=0)), ("EALIGN", "tkphi_quant_attention", dict(att__out=8196)), ("EALIGN", "tkphi_quant_attention", dict(att__lse=4097)),
        ("EINVAL", "tkphi_quant_block_attention", dict(cfg__block=0)), ("EINVAL", "tkphi_quant_block_attention", dict(cfg__last_blocks=0)),
        ("EUNSUPPORTED", "tkphi_quant_block_attention", dict(cfg__window=8)), ("EINVAL", "tkphi_quant_block_attention", dict(codes__M=0)),
        ("EINVAL", "tkphi_quant_read", dict(read__k=0, read__v=0)), ("EALIGN", "tkphi_quant_read", dict(read__k=4104)), ("EALIGN", "tkphi_quant_read", dict(read__v_row=60)),
        ("EALIGN", "tkphi_quant_read", dict(read__k_head=32)),
    ]:
        assert status(call, **kw) == getattr(B, "TKPHI_" + want), (call, kw, B.tkphi_last_error())


def test_binding_refuses_tensors_of_another_form():
    K = torch.zeros(3, 2, 16, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    S = torch.zeros(3, 2, 16, 2, dtype=torch.uint8)
    cfg = B.make_paged_config(4, 2, 64, "bf16", 0.1, K, K)
    assert (cfg.stride_page, cfg.stride_head, cfg.stride_tok, cfg.kv_dtype) == (2048, 1024, 64, B.TKPHI_BF16)
    B.make_quant_pool(K, K, S, torch.zeros(3, 2, 1, 64, dtype=torch.bfloat16))
    for call in (lambda: B.make_paged_config(4, 2, 64, "f32", 0.1, K, K), lambda: B.make_paged_config(4, 2, 64, "bf16", 0.1, K, K.float()),
                 lambda: B.make_paged_config(4, 2, 64, "bf16", 0.1, K.bfloat16(), K), lambda: B.make_pool(K, K), lambda: B.make_quant_pool(K.bfloat16(), K.bfloat16(), S),
                 lambda: B.make_quant_pool(K, K[:2], S), lambda: B.make_quant_pool(K, K, S.int()), lambda: B.make_quant_pool(K, K, S[:, :1]),
                 lambda: B.make_quant_pool(K, K, S.transpose(1, 2).contiguous().transpose(1, 2)), lambda: B.make_quant_pool(K, K, S, torch.zeros(3, 2, 1, 64)),
                 lambda: B.make_quant_pool(K, K.transpose(1, 2).contiguous().transpose(1, 2), S),
                 lambda: B.make_head_norms(torch.ones(1, 4, 64), None, 1e-6), lambda: B.make_head_norms(torch.ones(64), torch.ones(64).bfloat16(), 1e-6),
                 lambda: B.make_head_norms(torch.ones(64).half(), None, 1e-6), lambda: B.make_head_norms(torch.ones(128)[::2], None, 1e-6),
                 lambda: B.make_read_rows(None, None), lambda: B.make_read_rows(torch.zeros(3, 2, 64), None),
                 lambda: B.make_read_rows(torch.zeros(3, 2, 64).bfloat16(), torch.zeros(4, 2, 64).bfloat16()), lambda: B.make_read_rows(torch.zeros(2, 64).bfloat16(), None)):
        with pytest.raises(ValueError):
            call()


def test_calls_refuse_tensors_that_do_not_fit_config_and_step():
    K = torch.zeros(3, 2, 16, 64, dtype=torch.uint8).view(torch.float8_e4m3fn)
    cfg = B.make_paged_config(4, 2, 64, "bf16", 0.1, K, K, block=16, last_blocks=1)
    pool = B.make_quant_pool(K, K, torch.zeros(3, 2, 16, 2, dtype=torch.uint8), torch.zeros(3, 2, 1, 64, dtype=torch.bfloat16))
    plain = B.make_pool(K.bfloat16(), K.bfloat16())
    step = B.make_step(torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int32), 7, 7, 30)
    for thing in (step, pool, plain):
        thing.device = 0                     # (as if on a GPU: what is compared after the device)

    def rows(make, *shapes, **kw):
        io = make(*(None if s is None else torch.zeros(*s).bfloat16() for s in shapes), **kw)
        io.form = (*io.form[:2], 0)
        return io

    def refused(what, call, *args):
        with pytest.raises(ValueError, match=what):
            call(*args, 4096, 0, 0)

    def on_to_the_library(call, *args):      # (which refuses the workspace)
        with pytest.raises(B.TkphiError):
            call(*args, 4096, 0, 0)
    new = ((7, 4, 64), (7, 2, 64), (7, 2, 64), (7, 4, 64))
    ok = rows(B.make_new_rows, *new)

    def norms(*a, **kw):
        n = B.make_head_norms(*a, 1e-6, **kw)
        n.device = 0
        return n
    on_to_the_library(B.tkphi_quant_append, cfg, step, pool, ok, None)
    for good_norms in (norms(None, None), norms(torch.ones(64).bfloat16(), None), norms(torch.ones(4, 64).bfloat16(), torch.ones(2, 64).bfloat16(), offset=1.0),
                       norms(None, torch.ones(64).bfloat16())):
        on_to_the_library(B.tkphi_quant_append, cfg, step, pool, ok, good_norms)
    for bad in (norms(torch.ones(64), None), norms(torch.ones(128).bfloat16(), None), norms(torch.ones(2, 64).bfloat16(), None), norms(None, torch.ones(4, 64).bfloat16())):
        refused("norms", B.tkphi_quant_append, cfg, step, pool, ok, bad)
    away = norms(torch.ones(64).bfloat16(), None)
    away.device = 1
    refused("GPU 1", B.tkphi_quant_append, cfg, step, pool, ok, away)
    refused("pool", B.tkphi_norm_append, cfg, step, plain, ok, norms(None, None))       # (a config of codes with a pool of rows)
    refused("7", B.tkphi_quant_append, cfg, step, pool, rows(B.make_new_rows, *((6, *s[1:]) for s in new)), None)
    for call in (B.tkphi_quant_attention, B.tkphi_quant_block_attention):
        on_to_the_library(call, cfg, step, pool, rows(B.make_attention_rows, (7, 4, 64), (7, 4, 64)))
        refused("heads", call, cfg, step, pool, rows(B.make_attention_rows, (7, 2, 64), (7, 2, 64)))
        with pytest.raises(Exception):       # (a pool of another kind: no such struct)
            call(cfg, step, plain, rows(B.make_attention_rows, (7, 4, 64), (7, 4, 64)), 4096, 0, 0)
    on_to_the_library(B.tkphi_quant_read, cfg, step, pool, rows(B.make_read_rows, (7, 2, 64), None))
    refused("heads", B.tkphi_quant_read, cfg, step, pool, rows(B.make_read_rows, (7, 4, 64), None))
    refused("6 rows", B.tkphi_quant_read, cfg, step, pool, rows(B.make_read_rows, (6, 2, 64), (6, 2, 64)))


def test_oracle_on_cases_by_hand():
    x = np.array([[448.0, 1.0, -0.4375, 2.0 ** -9], [0.0, 0.0, 0.0, 0.0], [449.0, 0.0, 0.0, 17.0], [np.inf, np.nan, 3.0, -1.0]])
    codes, b = O.quantise(x)
    assert b.tolist() == [127, 10, 128, 127 - 7]
    assert codes[0].tolist() == [448.0, 1.0, -0.4375, 2.0 ** -9] and codes[2].tolist() == [224.0, 0.0, 0.0, 8.0] and np.isnan(codes[3, :2]).all()
    assert codes[3, 2:].tolist() == [384.0, -128.0]
    # every number of e4m3 is itself, and what torch rounds to it is what the oracle does
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    every = every[np.isfinite(every)]
    assert np.array_equal(O.e4m3(every), every)
    y = np.random.default_rng(0).normal(size=100000) * np.exp2(np.random.default_rng(1).integers(-12, 7, 100000))
    y = np.clip(y, -448, 448)
    assert np.array_equal(O.e4m3(y.astype(np.float32).astype(np.float64)), torch.from_numpy(y.astype(np.float32)).to(torch.float8_e4m3fn).double().numpy())
    n = O.head_norm(np.array([[3.0, 4.0]]), np.array([[1.0, 0.0]]), 0.0, 1.0)
    assert np.allclose(n, np.array([[6.0, 4.0]]) / np.sqrt(12.5))


def test_paged_cache_of_codes():
    c = PagedCache(4, 2, 64, 5, 16, 3, 40, 64, block=16, last_blocks=1, device="cpu", codes=True, norms=(torch.ones(64).bfloat16(), None, 1e-6))
    assert c.K.dtype == torch.float8_e4m3fn and c.scales.shape == (5, 2, 16, 2) and c.M.dtype == torch.bfloat16 and c.norms.eps > 0
    with pytest.raises(ValueError):
        PagedCache(4, 2, 64, 5, 16, 3, 40, 64, dtype="f32", device="cpu", codes=True)
    c.begin_step({"a": 17})
    c.end_step()
    with pytest.raises(ValueError):
        c.read("a", torch.zeros(16, 2, 64).bfloat16(), None)
    with pytest.raises(ValueError):
        PagedCache(4, 2, 64, 5, 16, 3, 40, 64, device="cpu").read("a", None, None)
