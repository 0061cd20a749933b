"""The calls on the paged cache refuse what the host can see to be wrong before any launch; their oracle on small cases."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2604_05438_amd import binding as B


def good(**kw):
    cfg = B.tkphi_paged_config(32, 8, 64, B.TKPHI_BF16, 0.125, 32, 8 * 32 * 64, 32 * 64, 64, 0, 64, 0, 16, 1, 2, 8, 0)
    step = B.tkphi_step(4096, 4096, 3, 10, 20, 12, 300, 0)
    pool = B.tkphi_kv_pool(4096, 8192, 16384, 40, 0)
    new = B.tkphi_new_rows(4096, 4096, 4096, 4096, 4096, 2048, 64, 512, 64, 512, 64, 2048, 64)
    att = B.tkphi_attention_rows(4096, 8192, 4096, 2048, 64, 2048, 64)
    for name, value in kw.items():
        where, field = name.split("__")
        setattr({"cfg": cfg, "step": step, "pool": pool, "new": new, "att": att}[where], field, value)
    return cfg, step, pool, new, att


CALLS = ("tkphi_kv_append", "tkphi_paged_attention", "tkphi_block_attention")


def status(call, ws=4096, short=0, **kw):
    cfg, step, pool, new, att = good(**kw)
    size = B.tkphi_paged_workspace_bytes(good()[0], good()[1])
    return getattr(B.lib(), call)(cfg, step, pool, new if call == "tkphi_kv_append" else att, ws, size - short, None)


EVERY = [
    ("EINVAL", dict(cfg__kv_dtype=2)), ("ESHAPE", dict(cfg__n_q_heads=30)), ("ESHAPE", dict(cfg__n_q_heads=72)), ("ESHAPE", dict(cfg__n_kv_heads=0)),
    ("ESHAPE", dict(cfg__d_head=96)), ("EINVAL", dict(cfg__score_scale=0.0)), ("EINVAL", dict(cfg__score_scale=float("nan"))),
    ("EINVAL", dict(cfg__score_scale=float("inf"))), ("EINVAL", dict(cfg__score_scale=-1.0)), ("ESHAPE", dict(cfg__page_tokens=0)),
    ("EALIGN", dict(cfg__stride_tok=60)), ("EALIGN", dict(cfg__stride_tok=32)), ("EALIGN", dict(cfg__stride_head=-64)), ("EALIGN", dict(cfg__stride_page=4)),
    ("EINVAL", dict(cfg__window=-1)), ("ESHAPE", dict(cfg__rot_dim=24)), ("ESHAPE", dict(cfg__rot_dim=80)), ("ESHAPE", dict(cfg__rot_adjacent=2)),
    ("ESHAPE", dict(cfg__block=8)), ("ESHAPE", dict(cfg__block=64)), ("EINVAL", dict(cfg__first_blocks=-1)), ("EINVAL", dict(cfg__top_blocks=2000)),
    ("EINVAL", dict(cfg__workgroups=5000)), ("EINVAL", dict(step__n_seqs=-1)), ("ESHAPE", dict(step__n_seqs=70000)), ("EINVAL", dict(step__rows=-1)),
    ("EINVAL", dict(step__reserved=1)), ("ESHAPE", dict(step__n_seqs=60000, step__max_len=1 << 30)), ("EINVAL", dict(step__seqs=0)), ("EALIGN", dict(step__seqs=4100)),
    ("EINVAL", dict(step__pages=0)), ("EINVAL", dict(step__max_pages=0)), ("EALIGN", dict(step__pages=4098)), ("EINVAL", dict(pool__K=0)), ("EALIGN", dict(pool__V=8200)),
    ("EINVAL", dict(pool__n_pages=0)), ("EINVAL", dict(pool__n_pages=-3)), ("EINVAL", dict(pool__reserved=1)),
]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("want,kw", EVERY)
def test_refusals_of_every_call(call, want, kw):
    assert status(call, **kw) in (getattr(B, "TKPHI_" + want), B.TKPHI_EWORKSPACE if "step__n_seqs" in kw else 99), B.tkphi_last_error()
    assert B.tkphi_last_error() != ""


@pytest.mark.parametrize("want,call,kw", [
    ("EINVAL", 0, dict(new__k=0)), ("EALIGN", 0, dict(new__v=4104)), ("EINVAL", 0, dict(new__q=0)), ("EINVAL", 0, dict(new__q_rot=0)),
    ("EALIGN", 0, dict(new__k_row=60)), ("EALIGN", 0, dict(new__q_head=32)), ("EINVAL", 0, dict(new__inv_freq=0)), ("EALIGN", 0, dict(new__inv_freq=4100)),
    ("EINVAL", 0, dict(pool__M=0)), ("EALIGN", 0, dict(pool__M=4104)),
    ("EINVAL", 1, dict(att__q=0)), ("EINVAL", 1, dict(att__out=0)), ("EALIGN", 1, dict(att__out=8196)), ("EALIGN", 1, dict(att__lse=4097)),
    ("EALIGN", 1, dict(att__out_row=65)), ("EALIGN", 1, dict(att__q_row=-64)),
    ("EINVAL", 2, dict(cfg__block=0)), ("EINVAL", 2, dict(cfg__last_blocks=0)), ("EUNSUPPORTED", 2, dict(cfg__window=8)), ("EINVAL", 2, dict(pool__M=0)),
])
def test_refusals(want, call, kw):
    assert status(CALLS[call], **kw) == getattr(B, "TKPHI_" + want), B.tkphi_last_error()


@pytest.mark.parametrize("call", CALLS)
def test_workspace_refusals_and_empty_steps(call):
    assert status(call, ws=None) == B.TKPHI_EWORKSPACE
    assert status(call, ws=4100) == B.TKPHI_EWORKSPACE
    assert status(call, short=256) == B.TKPHI_EWORKSPACE
    for kw in (dict(step__n_seqs=0, step__seqs=0), dict(step__rows=0), dict(step__max_new=0), dict(step__max_len=0)):
        assert status(call, pool__n_pages=0, **kw) == B.TKPHI_OK
    cfg, step, pool, new, att = good()
    f = getattr(B.lib(), call)
    assert f(None, step, pool, new if call == CALLS[0] else att, 4096, 1 << 30, None) == B.TKPHI_EINVAL
    assert f(cfg, step, None, new if call == CALLS[0] else att, 4096, 1 << 30, None) == B.TKPHI_EINVAL
    assert f(cfg, step, pool, None, 4096, 1 << 30, None) == B.TKPHI_EINVAL


def test_workspace_serves_smaller_steps():
    import random
    r = random.Random(4)
    for _ in range(600):
        hkv = r.choice([1, 2, 8])
        cfg = B.tkphi_paged_config(hkv * r.choice([1, 3, 7, 8]), hkv, r.choice([64, 128]), r.choice([0, 1]), 0.1, 64, 1 << 20, 1 << 14, 1 << 10, 0, 0, 0,
                                   r.choice([0, 16, 64]), r.randint(0, 3), r.randint(1, 3), r.randint(0, 100), r.choice([0, 0, 5]))
        n, rows, new, length = r.randint(1, 300), r.randint(1, 3000), r.randint(1, 3000), r.randint(1, 200000)
        big = B.tkphi_paged_workspace_bytes(cfg, B.tkphi_step(16, 16, n, 9, rows, new, length, 0))
        assert big > 0, B.tkphi_last_error()
        for _ in range(5):
            small = B.tkphi_step(16, 16, r.randint(0, n), 9, r.randint(0, rows), r.randint(0, new), r.randint(0, length), 0)
            assert 0 < B.tkphi_paged_workspace_bytes(cfg, small) <= big


def test_binding_refuses_tensors_of_another_form():
    K = torch.zeros(3, 2, 16, 64)
    with pytest.raises(ValueError):
        B.make_paged_config(4, 2, 64, "bf16", 0.1, K, K)
    with pytest.raises(ValueError):
        B.make_paged_config(4, 2, 64, "f32", 0.1, K, K.transpose(1, 2))
    with pytest.raises(ValueError):
        B.make_paged_config(4, 2, 128, "f32", 0.1, K, K)
    cfg = B.make_paged_config(4, 2, 64, "f32", 0.1, K.transpose(1, 2).contiguous().transpose(1, 2), K.transpose(1, 2).contiguous().transpose(1, 2))
    assert (cfg.stride_page, cfg.stride_head, cfg.stride_tok) == (2048, 64, 128)
    seqs, pages = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, 5, dtype=torch.int32)
    for a, b in ((seqs.long(), pages), (seqs, pages.long()), (seqs[:1], pages), (seqs[:, :3], pages), (seqs, pages.T), (seqs, pages[:, ::2])):
        with pytest.raises(ValueError):
            B.make_step(a, b, 2, 1, 10)
    with pytest.raises(ValueError):
        B.make_pool(K, K, torch.zeros(3, 2, 1, 32))
    q, k = torch.zeros(2, 4, 64), torch.zeros(2, 2, 64)
    for bad in (dict(v=k[:1]), dict(q=q.bfloat16()), dict(q_rot=q[:, :3]), dict(k=k[..., ::2]), dict(inv_freq=torch.zeros(8))):
        with pytest.raises(ValueError):
            B.make_new_rows(**{**dict(q=q, k=k, v=k, q_rot=q), **bad})
    for bad in (dict(out=q.bfloat16()), dict(out=q[:, :2]), dict(lse=torch.zeros(2, 3)), dict(lse=torch.zeros(4, 2).T), dict(q=q[0])):
        with pytest.raises(ValueError):
            B.make_attention_rows(**{**dict(q=q, out=q), **bad})


def test_oracle_on_a_case_by_hand():
    # two tokens, scores 0 and log 3: weights 1/4 and 3/4
    K = np.array([[[[0.0, 0.0], [0.0, 0.0]]]])
    V = np.array([[[[4.0, 0.0], [0.0, 8.0]]]])
    K[0, 0, 1, 0] = np.log(3.0)
    q = np.array([[[1.0, 0.0]]])
    y, lse, spread, _ = O.paged_attention(q, K, V, [0], 1, 1, 1.0)[0][0]
    assert np.allclose(y, [1.0, 6.0]) and np.isclose(lse, np.log(4.0))
    y, lse, _, _ = O.paged_attention(q, K, V, [0], 1, 1, 1.0, window=1)[0][0]
    assert np.allclose(y, [0.0, 8.0]) and np.isclose(lse, np.log(3.0))
    assert np.allclose(O.rotate(np.array([[1.0, 0.0, 5.0]]), 1, np.array([np.pi / 2]), False), [[0.0, 1.0, 5.0]])
    M = np.array([[[1.0], [3.0]], [[3.0], [2.0]], [[0.0], [0.0]]])
    assert O.pick_blocks(np.array([[1.0]]), M, [0, 1, 2], 2, 4, 11, 0, 1, 1) == [1, 5]
    assert O.pick_blocks(np.array([[-1.0], [0.5]]), M, [0, 1, 2], 2, 4, 11, 1, 1, 2) == [0, 1, 2, 5]


def test_calls_refuse_tensors_that_do_not_fit_config_and_step(monkeypatch):
    """Rows, heads, channels, type, pool and device are compared before anything is launched.  (On the CPU what fits ends at the device.)"""
    from paper_2604_05438_amd.paged import PagedCache
    monkeypatch.setattr(B, "current_stream_ptr", lambda: 0)
    c = PagedCache(4, 2, 64, 5, 16, 3, 40, 64, block=16, last_blocks=1, device="cpu")
    c.begin_step({"a": 5, "b": 2})

    def rows(n=7, heads=4, d=64, dtype=torch.bfloat16):
        return torch.zeros(n, heads, d, dtype=dtype)

    def refused(what, call, *args):
        with pytest.raises(ValueError, match=what):
            call(*args)
    for call in (c.attend, c.attend_blocks):
        refused("7", call, rows(6), rows(6))
        refused("heads", call, rows(heads=2), rows(heads=2))
        refused("channels", call, rows(d=128), rows(d=128))
        refused("storage type", call, rows(dtype=torch.float32), rows(dtype=torch.float32))
        refused("storage type", call, rows(dtype=torch.float16), rows(dtype=torch.float16))
        refused("not on a GPU", call, rows(), rows())
        refused("not on a GPU", call, rows(9), rows(9))
        refused("GPUs", call, rows(), rows().to("meta"))
    kv = dict(heads=2)
    refused("7", c.append, rows(6), rows(6, **kv), rows(6, **kv), rows(6))
    refused("heads", c.append, rows(heads=2), rows(**kv), rows(**kv), rows(heads=2))
    refused("heads", c.append, rows(), rows(), rows(), rows())
    refused("storage type", c.append, *(rows(heads=h, dtype=torch.float32) for h in (4, 2, 2, 4)))
    refused("not on a GPU", c.append, rows(), rows(**kv), rows(**kv), rows())
    refused("not on a GPU", c.append, None, rows(**kv), rows(**kv), None)
    # the pool, its means and the angles
    K = torch.zeros(5, 2, 32, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="V"):
        B.make_pool(K, K[:4])
    with pytest.raises(ValueError, match="V"):
        B.make_pool(K, K.transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(ValueError, match="V"):
        B.make_pool(K, K.float())
    cfg = B.make_paged_config(4, 2, 64, "bf16", 0.1, K, K, rot_dim=64, block=16, last_blocks=1)
    seqs, pages = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int32)
    step = B.make_step(seqs, pages, 7, 7, 60)
    pool = B.make_pool(K, K, torch.zeros(5, 2, 2, 64, dtype=torch.bfloat16))
    for thing in (step, pool):
        thing.device = 0                     # (as if on a GPU: what is compared after the device)

    def io(angles):
        x = B.make_new_rows(rows(), rows(**kv), rows(**kv), rows(), inv_freq=torch.zeros(angles, dtype=torch.float64))
        x.form = (*x.form[:2], 0)
        return x
    refused("inv_freq", B.tkphi_kv_append, cfg, step, pool, io(31), 4096, 0, 0)
    with pytest.raises(B.TkphiError):        # (as it should be: on to the library, which refuses the workspace)
        B.tkphi_kv_append(cfg, step, pool, io(32), 4096, 0, 0)
    for other in (torch.zeros(5, 2, 16, 64, dtype=torch.bfloat16), K.transpose(1, 2).contiguous().transpose(1, 2), torch.zeros(5, 4, 32, 64, dtype=torch.bfloat16)):
        bad = B.make_pool(other, other)
        bad.device = 0
        refused("pool", B.tkphi_kv_append, cfg, step, bad, io(32), 4096, 0, 0)
    bad = B.make_pool(K, K, torch.zeros(5, 2, 1, 64, dtype=torch.bfloat16))
    bad.device = 0
    refused("blocks per page", B.tkphi_kv_append, cfg, step, bad, io(32), 4096, 0, 0)


@pytest.mark.parametrize("dtype,hq,hkv,d,step,most", [
    # (sequences, rows, max_new, max_len); two partials per workgroup: as many of those as the step has units of 64 (bf16 single tokens: 128) cached tokens, or fit the GPU
    (0, 1, 1, 64, (1, 1, 1, 4096), 64 * 2 * 16),
    (0, 1, 1, 64, (1, 1, 1, 100), 2 * 2 * 16),
    (1, 32, 8, 64, (1, 1, 1, 4096), 8 * 32 * 2 * 16),
    (1, 24, 8, 128, (32, 32, 1, 65000), 512 * 2 * 16),
    (0, 24, 8, 128, (4, 1200, 300, 16000), 512 * 2 * 32),
    (1, 24, 8, 128, (1, 2048, 2048, 32000), 256 * 2 * 256),
    (1, 32, 8, 64, (4, 8000, 4000, 4000), 768 * 2 * 128),
])
def test_workspace_is_what_the_steps_need(dtype, hq, hkv, d, step, most):
    cfg = B.tkphi_paged_config(hq, hkv, d, dtype, 0.1, 64, 1 << 20, 1 << 14, 1 << 10, 0)
    n, rows, new, length = step
    items = rows * hq // hkv // 16 + n
    size = B.tkphi_paged_workspace_bytes(cfg, B.tkphi_step(16, 16, n, 9, rows, new, length, 0))
    assert 0 < size <= most * (d + 2) * 4 + items * 16 + 4096 + 32768 + 6 * 256
