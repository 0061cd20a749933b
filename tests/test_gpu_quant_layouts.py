"""The calls on the cache in 8 bits on pools whose tokens are further apart than their heads are long, and on pools beyond 2^32 bytes."""
import pytest
import torch

import paged_utils as P
import quant_utils as Q
import test_gpu_quant_append as A
from paper_2604_05438_amd import binding as B

pytestmark = pytest.mark.gpu


class Padded(Q.Step):
    """Tokens outermost, `pad` more heads per token that nobody reads or writes (codes that are no numbers)"""

    def __init__(self, *a, pad=1, **kw):
        super().__init__(*a, heads_first=False, **kw)
        self.pad = pad
        self.room = {n: self.padded(getattr(self, n)) for n in ("K8", "V8")}
        self.K8, self.V8 = (self.seen(x) for x in self.room.values())

    def padded(self, x):
        room = torch.full((self.n_pages, self.page, self.hkv + self.pad, self.d), 0x7f, dtype=torch.uint8).view(torch.float8_e4m3fn)
        room.view(torch.uint8)[:, :, :self.hkv] = x.transpose(1, 2).view(torch.uint8)
        return room

    def seen(self, room):
        return room[:, :, :self.hkv].transpose(1, 2)

    def upload(self):
        super().upload()
        self.dev_room = {n: x.cuda() for n, x in self.room.items()}
        self.dev.update({n: self.seen(x) for n, x in self.dev_room.items()})
        return self

    def check_padding(self):
        for x in self.dev_room.values():
            assert (x.view(torch.uint8)[:, :, self.hkv:] == 0x7f).all()


def attend(st, window=0, workgroups=0):
    st.upload()
    cfg = st.config(window=window, workgroups=workgroups)
    out, lse = st.call(B.tkphi_quant_attention, cfg)
    P.check(st, out, lse, P.attention_oracle(st, window=window))
    return cfg


@pytest.mark.parametrize("heads,lens", [((32, 8, 64), [(0, 1), (31, 1), (500, 1), (2000, 2), (63, 2)]), ((4, 4, 64), [(0, 8), (100, 5), (900, 3), (3, 0)]), ((16, 2, 64), [(700, 1), (64, 1)])])
@pytest.mark.parametrize("page,pad", [(16, 1), (8, 2), (104, 5)])
def test_two_heads_per_item_of_padded_tokens(heads, lens, page, pad):
    """Pairs of heads where the next token is not right behind the last head"""
    for workgroups, window in ((0, 0), (3, 0), (0, 40)):
        cfg = attend(Padded(*heads, lens, page, pad=pad, seed=8, slack_rows=1), window, workgroups)
        assert (cfg.stride_head, cfg.stride_tok) == (64, 64 * (heads[1] + pad))
    st = Padded(*heads, lens, page, pad=pad, seed=9, garbage=float("nan"))
    st.table[0, 0] = -1
    attend(st)


@pytest.mark.parametrize("heads", [(32, 8, 64), (6, 3, 64), (10, 2, 128)])
@pytest.mark.parametrize("page", [16, 100])
def test_all_calls_on_padded_tokens(heads, page):
    for lens in ([(300, 1), (40, 2)], [(77, 3), (0, 4), (500, 4)], [(70, 60), (0, 130)]):
        attend(Padded(*heads, lens, page, seed=5))
    attend(Padded(*heads, [(60, 1)] * 70, page, seed=5, pad=3))
    st = Padded(*heads, [(0, 40), (33, 1), (5, 30)], page, seed=2)
    A.check(st, 64)
    st.check_padding()
    A.read(Padded(*heads, [(0, 40), (33, 1), (5, 130)], page, seed=2), layout="heads")
    if page % 16:
        return
    st = Padded(*heads, [(15, 1), (5, 40)], page, block=16, seed=2)
    A.check(st, 64, norm=None)
    st.check_padding()
    st = Padded(*heads, [(700, 1), (90, 3)], page, block=16, seed=3).upload()
    out, _ = st.call(B.tkphi_quant_block_attention, st.config(first_blocks=1, last_blocks=2, top_blocks=5))
    P.check(st, out, None, P.block_oracle(st, 1, 2, 5))


def plain(x):
    return x.view(torch.uint8) if x.element_size() == 1 else x


class Far:
    """The device's pools of a step with every used page moved to a place of its own in pools of more than 2^32 bytes, first and last ones in turn"""

    def __init__(self, st, heads_first):
        self.st, self.n_pages = st, (1 << 32) // (st.hkv * st.page * st.d) + 40
        used = sorted({int(p) for p in st.table.reshape(-1) if p >= 0})
        self.used = torch.tensor(used, device="cuda")
        self.place = torch.tensor([self.n_pages - 1 - 3 * i if i % 2 else 2 * i for i in range(len(used))], device="cuda")
        back = dict(zip(used, self.place.tolist()))
        self.table = torch.tensor([[back.get(int(p), -1) for p in row] for row in st.table], dtype=torch.int32, device="cuda")
        self.big = {}
        for n in ("K8", "V8", "S", "M"):
            x = st.dev[n]
            if x is None:
                self.big[n] = None
                continue
            move = n in ("K8", "V8") and not heads_first
            x = plain(x.transpose(1, 2) if move else x)
            big = torch.zeros(self.n_pages, *x.shape[1:], device="cuda", dtype=x.dtype)
            big[self.place] = x[self.used]
            big = big.view(st.dev[n].dtype)
            self.big[n] = big.transpose(1, 2) if move else big
        assert self.big["K8"].nelement() > 1 << 32

    def pages_of(self, n):
        """The used pages, in the small pool's order; all others are still zeros"""
        x = plain(self.big[n])
        got = x[self.place].clone()
        x[self.place] = 0
        assert not x.any()
        x[self.place] = got
        return got

    def args(self, **kw):
        st = self.st
        cfg = B.make_paged_config(st.hq, st.hkv, st.d, "bf16", st.d ** -0.5, self.big["K8"], self.big["V8"], block=st.block, **kw)
        step = B.make_step(st.dev["seqs"], self.table, st.rows, st.max_new, st.max_len)
        return cfg, step, B.make_quant_pool(self.big["K8"], self.big["V8"], self.big["S"], self.big["M"])


def on(cfg, step, call, pool, *io):
    ws = B.alloc_paged_workspace(B.tkphi_paged_workspace_bytes(cfg, step))
    call(cfg, step, pool, *io, ws.data_ptr(), ws.numel(), B.current_stream_ptr())
    assert B.tkphi_read_device_status(ws.data_ptr(), B.current_stream_ptr()) == 0


@pytest.mark.parametrize("heads_first", [True, False])
def test_append_blocks_and_read_beyond_32_bits(heads_first):
    """As in a small pool, to the bit"""
    lens = [(90, 40), (60, 5), (15, 1)]
    st = Q.Step(4, 2, 64, lens, 16, heads_first=heads_first, block=16, seed=6).upload()
    far = Far(st, heads_first)
    gen = torch.Generator(device="cuda").manual_seed(5)
    qkv = torch.randn(st.rows, 8, 64, generator=gen, device="cuda").bfloat16()
    freq = torch.from_numpy(A.inv_freq(64)).cuda()
    kw = dict(rot_dim=64, first_blocks=1, last_blocks=1, top_blocks=2)
    results = []
    for cfg, step, pool in ((st.config(**kw), st.step(), st.pool()), far.args(**kw)):
        q_rot, out = torch.full((2, st.rows, 4, 64), 7.0, device="cuda", dtype=torch.bfloat16)
        back = torch.full((2, st.rows, 2, 64), 7.0, device="cuda", dtype=torch.bfloat16)
        on(cfg, step, B.tkphi_quant_append, pool, B.make_new_rows(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], q_rot, inv_freq=freq), None)
        on(cfg, step, B.tkphi_quant_block_attention, pool, B.make_attention_rows(q_rot, out))
        on(cfg, step, B.tkphi_quant_read, pool, B.make_read_rows(back[0], back[1]))
        results.append((q_rot, out, back))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert (results[0][1] != 7).any()
    for n in ("K8", "V8", "S", "M"):
        assert torch.equal(far.pages_of(n), plain(st.dev[n])[far.used]), n


@pytest.mark.parametrize("lens", [[(90, 1), (60, 2), (300, 1)], [(90, 6), (60, 5)], [(90, 40), (10, 20)]])
def test_attention_beyond_32_bits_with_tokens_outermost(lens):
    """Pairs of heads, heads by themselves, chunks"""
    st = Q.Step(8, 2, 64, lens, 16, heads_first=False, seed=6).upload()
    far = Far(st, False)
    want = P.attention_oracle(st)
    results = []
    for cfg, step, pool in ((st.config(), st.step(), st.pool()), far.args()):
        out, lse = torch.full((st.rows, 8, 64), 7.0, device="cuda", dtype=torch.bfloat16), torch.full((st.rows, 8), 7.0, device="cuda")
        on(cfg, step, B.tkphi_quant_attention, pool, B.make_attention_rows(st.dev["q"], out, lse))
        P.check(st, out.double().cpu().numpy(), lse.double().cpu().numpy(), want)
        results.append((out, lse))
    assert all(torch.equal(a, b) for a, b in zip(*results))
