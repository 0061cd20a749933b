"""The calls on the paged key/value cache whose speed this framework is held to: tkphi_kv_append (rotates new keys and
queries, writes keys and values to their pages, and the mean key of every block that fills up), tkphi_paged_attention
(new tokens over everything cached) and tkphi_block_attention (new tokens over the blocks whose mean keys score highest).
Where `own` is false, run() computes the same from elementary torch operations.

A case is a dict of
  op          "append", "attend" or "blocks"
  dtype       storage of q, k, v and the cache: "bf16" or "f32"
  hq, hkv, d  query heads, KV heads, head dimension
  seqs, ctx_min, ctx_max, new_min, new_max
              sequences; each has ctx_min..ctx_max tokens in the cache and brings new_min..new_max more
  page        tokens per page; pages lie in the pool in random order
  heads_first pages are [head][token][channel]; else [token][head][channel]
  block       tokens per block (append: 0 keeps no means)
  first, last, top
              blocks: those every query sees at either end, and those it retrieves
  window      attend: tokens a query sees back (0: all); pages behind every window are absent
  rot, adjacent
              append: rotated channels; pairs (2j, 2j + 1) instead of (j, j + rot / 2)

Values: queries, keys, values ~ N(0, 1), four channels of every KV head five times that in the keys, and 16 keys of
every sequence and KV head along one of its queries (cosine 0.8): sharp peaks on top of diffuse mass.
"""
import math
import random

import torch

own = False

HEADS = {"1b": (32, 8, 64), "3b": (24, 8, 128), "head": (1, 1, 64)}
NEEDLES = 16


def _case(name, op, dtype="bf16", model="3b", seqs=1, ctx=(0, 0), new=(1, 1), page=16, heads_first=True, block=0, first=0, last=0, top=0,
          window=0, rot=None, adjacent=False):
    hq, hkv, d = HEADS[model] if isinstance(model, str) else model
    c = dict(op=op, dtype=dtype, hq=hq, hkv=hkv, d=d, seqs=seqs, ctx_min=ctx[0], ctx_max=ctx[1], new_min=new[0], new_max=new[1], page=page,
             heads_first=heads_first, block=block, first=first, last=last, top=top, window=window, rot=d if rot is None else rot,
             adjacent=adjacent)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one fp32 head (a debugging or accuracy run)
        _case("append_f32_head", "append", "f32", "head", ctx=(4000, 4000)),
        # a serving step: one token each of 64 running sequences
        _case("append_3b_batch64", "append", seqs=64, ctx=(500, 16000), block=16),
        # ragged chunks of several prompts, another layout, rotation of half of the channels in adjacent pairs
        _case("append_1b_chunks", "append", model="1b", seqs=5, ctx=(0, 3000), new=(100, 900), page=64, heads_first=False, block=32, rot=32,
              adjacent=True),
        # a long prompt in one chunk
        _case("append_3b_prompt", "append", new=(16001, 16001), page=64, block=32),
        # interactive use: one token over a short context; one fp32 head, and the 1B layer
        _case("attend_f32_head", "attend", "f32", "head", ctx=(4095, 4095)),
        _case("attend_1b_4k", "attend", model="1b", ctx=(4001, 4001)),
        # a serving step of 32 running sequences, and one that checks five drafted tokens of each of 8
        _case("attend_3b_batch32", "attend", seqs=32, ctx=(2000, 65000)),
        _case("attend_3b_draft", "attend", seqs=8, ctx=(1000, 16000), new=(5, 5), page=32),
        # a chunk of a long prompt, and short prompts of a 1B model from their start
        _case("attend_3b_chunk", "attend", ctx=(30000, 30000), new=(2048, 2048), page=64),
        _case("attend_1b_prompts", "attend", model="1b", seqs=4, new=(700, 4000), page=64, heads_first=False),
        # sparse steps: one token over 128K tokens, and 16 sequences
        _case("blocks_3b_128k", "blocks", ctx=(131000, 131000), page=64, block=32, first=1, last=2, top=61),
        _case("blocks_1b_batch16", "blocks", model="1b", seqs=16, ctx=(16000, 65000), page=32, block=32, first=1, last=2, top=45),
    ]


def draw(rng):
    def log(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    op = rng.choice(["append", "attend", "attend", "blocks"])
    dtype = "f32" if rng.random() < 0.15 else "bf16"
    model = rng.choice(["1b", "3b", (8, 8, 64), (40, 8, 128), (14, 2, 64), (8, 1, 128), (12, 4, 128)])
    hq, hkv, d = HEADS[model] if isinstance(model, str) else model
    kw = dict(heads_first=rng.random() < 0.5, page=rng.choice([16, 32, 64, 128, 256]))
    if op == "append":
        seqs = log(1, 64)
        new = log(1, max(1, 16000 // seqs))
        ctx = log(1, 16000)
        if rng.random() < 0.6:
            kw["block"] = rng.choice([b for b in (16, 32, 64) if kw["page"] % b == 0])
        else:
            kw["page"] = rng.choice([kw["page"], 24, 100])
        return _case(None, op, dtype, model, seqs, (ctx // 8, ctx), (max(1, new // 3), new), rot=rng.choice([d, d, d // 2, 16]),
                     adjacent=rng.random() < 0.4, **kw)
    if op == "blocks":
        kw["block"] = rng.choice([b for b in (16, 32, 64) if kw["page"] % b == 0])
        ctx = log(1000, 131000)
        seqs = log(1, max(1, min(16, 500000 // ctx)))
        return _case(None, op, dtype, model, seqs, (ctx // 4, ctx), (1, rng.choice([1, 1, 1, 4])), first=rng.randint(0, 4), last=rng.randint(1, 4),
                     top=log(8, 128), **kw)
    if rng.random() < 0.5:      # single tokens and a few
        ctx, new = log(100, 65000), rng.choice([1, 1, 1, 2, 5, 8])
        seqs = log(1, max(1, min(64, 800000 // ctx)))
    else:                       # chunks and prompts
        ctx, new = rng.choice([0, log(1, 32000)]), log(16, 4000)
        seqs = log(1, 8)
    if dtype == "f32":
        ctx, seqs = min(ctx, 16000), min(seqs, 4)
    while seqs > 1 and seqs * hq * new * (ctx + new) > 1.2e9:
        seqs -= 1
    while hq * new * (ctx + new) > 1.2e9:
        new = new * 3 // 4
    if kw["page"] == 16 and rng.random() < 0.3:
        kw["page"] = rng.choice([24, 100])
    return _case(None, op, dtype, model, seqs, (ctx // 4, ctx), (max(1, new // 3), new), window=log(64, 8000) if rng.random() < 0.25 else 0, **kw)


# ---- what a program has in hand ------------------------------------------------------------------------------------------
def _lengths(c):
    """(tokens cached, tokens new) of every sequence"""
    r = random.Random(c["ctx_min"] * 1000003 + c["ctx_max"] * 17 + c["seqs"] * 5 + c["new_max"])
    return [(r.randint(c["ctx_min"], c["ctx_max"]), r.randint(c["new_min"], c["new_max"])) for _ in range(c["seqs"])]


def _dt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _inv_freq(c):
    return 500000.0 ** (-torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64) / c["rot"])


def _pages(c, gen):
    """Page ids [seqs][max_pages], -1 behind the end and behind every window; the pool's number of pages, and one that nobody has."""
    ps, lens = c["page"], _lengths(c)
    count = [-(-(n + m) // ps) for n, m in lens]
    n_pages = sum(count) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32).cpu()
    table, at = torch.full((c["seqs"], max(count)), -1, dtype=torch.int32), 0
    for i, (n, _) in enumerate(lens):
        table[i, :count[i]] = order[at:at + count[i]]
        at += count[i]
        if c["window"]:
            table[i, :max(0, n + 1 - c["window"]) // ps] = -1
    return table.cuda(), n_pages, int(order[-1])


def _pool(c, n_pages, gen, loud=None):
    shape = (n_pages, c["hkv"], c["page"], c["d"]) if c["heads_first"] else (n_pages, c["page"], c["hkv"], c["d"])
    x = torch.randn(shape, generator=gen, device="cuda", dtype=_dt(c))
    x = x if c["heads_first"] else x.transpose(1, 2)
    if loud is not None:
        x *= loud[:, None, :]
    return x


def prepare(case, seed):
    """A serving program's state in the middle of a step: the pool with the cached tokens, page table and lengths of the
    running sequences, the new tokens' rows, output buffers; with `own` the library's descriptors and workspace."""
    c = case
    hq, hkv, d, ps, dt, B = c["hq"], c["hkv"], c["d"], c["page"], _dt(c), c["block"]
    gen = torch.Generator(device="cuda").manual_seed((int(seed) * 7919 + 20260405) % (1 << 62))
    lens = _lengths(c)
    rows = sum(m for _, m in lens)
    first_row = [sum(m for _, m in lens[:i]) for i in range(len(lens))]
    seqs = torch.tensor([[n, m, r, 0] for (n, m), r in zip(lens, first_row)], dtype=torch.int32).cuda()
    pages, n_pages, spare = _pages(c, gen)
    seq_of = torch.repeat_interleave(torch.arange(c["seqs"]), torch.tensor([m for _, m in lens])).cuda()
    pos = (torch.arange(rows, device="cuda") - seqs[seq_of, 2] + seqs[seq_of, 0]).long()      # cache position of every new token
    loud = torch.ones(hkv, d, device="cuda", dtype=dt).scatter_(1, torch.rand(hkv, d, generator=gen, device="cuda").topk(4, dim=1).indices, 5.0)
    s = {"case": c, "rows": rows, "seqs": seqs, "pages": pages, "n_pages": n_pages, "seq_of": seq_of, "pos": pos,
         "max_new": max(m for _, m in lens), "max_len": max(n + m for n, m in lens),
         "K": _pool(c, n_pages, gen, loud), "V": _pool(c, n_pages, gen)}
    if c["op"] == "append":
        qkv = torch.randn(rows, hq + 2 * hkv, d, generator=gen, device="cuda", dtype=dt)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["q_rot"] = torch.empty(rows, hq, d, device="cuda", dtype=dt)
        s["inv_freq"] = _inv_freq(c)
        if B:
            s["M"] = torch.zeros(n_pages, hkv, ps // B, d, device="cuda", dtype=dt)
            done = [(i, b) for i, (n, m) in enumerate(lens) for b in range(n // B, (n + m) // B)]
            s["done"] = torch.tensor(done, dtype=torch.int64).reshape(-1, 2).cuda()     # (sequence, block) that fill up
    else:
        s["q"] = torch.randn(rows, hq, d, generator=gen, device="cuda", dtype=torch.float32)
        _needles(s, spare, gen)
        s["q"] = s["q"].to(dt)
        s["out"] = torch.empty(rows, hq, d, device="cuda", dtype=dt)
        if c["op"] == "attend":
            s["lse"] = torch.empty(rows, hq, device="cuda")
            s["row_at"] = torch.tensor([[r + min(i, m - 1) for i in range(s["max_new"])] for (_, m), r in zip(lens, first_row)]).cuda()
        else:
            s["M"] = s["K"].unflatten(2, (ps // B, B)).float().mean(3).to(dt).contiguous()
    s["own"] = _descriptors(s) if own else None
    return s


def _needles(s, spare, gen):
    """Sets up to 16 cached keys of every sequence and KV head along one of its queries (those of absent pages go to a spare one)."""
    c, (hq, hkv, d) = s["case"], (s["case"]["hq"], s["case"]["hkv"], s["case"]["d"])
    lens = _lengths(c)
    n, count = len(lens), min(NEEDLES, min(a + b for a, b in lens))
    length = (s["seqs"][:, 0] + s["seqs"][:, 1])[:, None].double()
    t = ((torch.arange(count, device="cuda") + torch.rand(n, count, generator=gen, device="cuda").double() * 0.99) * (length / count)).long()
    page = s["pages"].gather(1, t // c["page"]).long()
    page = torch.where(page < 0, spare, page)
    row = (s["seqs"][:, 2, None] + (torch.rand(n, count, generator=gen, device="cuda") * s["seqs"][:, 1, None] * 0.99).long()).long()
    G = hq // hkv
    head = torch.arange(hkv, device="cuda") * G + (torch.arange(count, device="cuda") % G)[:, None]
    along = torch.nn.functional.normalize(s["q"][row[:, :, None], head], dim=-1)              # [seqs][needles][hkv][d]
    side = torch.randn(n, count, hkv, d, generator=gen, device="cuda")
    side = torch.nn.functional.normalize(side - (side * along).sum(-1, keepdim=True) * along, dim=-1)
    s["K"][page[:, :, None], torch.arange(hkv, device="cuda"), (t % c["page"])[:, :, None]] = (math.sqrt(d) * (0.8 * along + 0.6 * side)).to(_dt(c))


def _descriptors(s):
    from paper_2604_05438_amd import binding as B
    c = s["case"]
    cfg = B.make_paged_config(c["hq"], c["hkv"], c["d"], c["dtype"], c["d"] ** -0.5, s["K"], s["V"], window=c["window"],
                              rot_dim=c["rot"] if c["op"] == "append" else 0, rot_adjacent=c["adjacent"], block=c["block"],
                              first_blocks=c["first"], last_blocks=c["last"], top_blocks=c["top"])
    step = B.make_step(s["seqs"], s["pages"], s["rows"], s["max_new"], s["max_len"])
    pool = B.make_pool(s["K"], s["V"], s.get("M"))
    if c["op"] == "append":
        io = B.make_new_rows(s["q"], s["k"], s["v"], s["q_rot"], inv_freq=s["inv_freq"])
    else:
        io = B.make_attention_rows(s["q"], s["out"], s.get("lse"))
    size = B.tkphi_paged_workspace_bytes(cfg, step)
    call = {"append": B.tkphi_kv_append, "attend": B.tkphi_paged_attention, "blocks": B.tkphi_block_attention}[c["op"]]
    return {"call": call, "cfg": cfg, "step": step, "pool": pool, "io": io, "ws": B.alloc_paged_workspace(size), "size": size,
            "stream": B.current_stream_ptr}


# ---- the operators ---------------------------------------------------------------------------------------------------------
def run(state):
    s, op = state, state["case"]["op"]
    if own:
        o = s["own"]
        o["call"](o["cfg"], o["step"], o["pool"], o["io"], o["ws"].data_ptr(), o["size"], o["stream"]())
        return _outputs(s)
    if op == "append":
        _append(s)
    elif op == "attend":
        _attend(s)
    else:
        _blocks(s)
    return _outputs(s)


def _outputs(s):
    names = {"append": ("q_rot", "K", "V", "M"), "attend": ("out", "lse"), "blocks": ("out",)}[s["case"]["op"]]
    return {n: s[n] for n in names if n in s}


def _rotate(x, cos, sin, c):
    """x [rows][heads][d] in the precision of cos, sin [rows][rot / 2]"""
    r, h = c["rot"], c["rot"] // 2
    cos, sin = cos[:, None], sin[:, None]
    if c["adjacent"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :h], x[..., h:r]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _append(s):
    c, dt = s["case"], _dt(s["case"])
    angle = s["pos"].double()[:, None] * s["inv_freq"]
    cos, sin = angle.cos().float(), angle.sin().float()
    s["q_rot"].copy_(_rotate(s["q"].float(), cos, sin, c).to(dt))
    page = s["pages"][s["seq_of"], s["pos"] // c["page"]].long()
    row = s["pos"] % c["page"]
    s["K"][page, :, row] = _rotate(s["k"].float(), cos, sin, c).to(dt)
    s["V"][page, :, row] = s["v"]
    if c["block"]:
        B, per = c["block"], c["page"] // c["block"]
        of, b = s["done"][:, 0], s["done"][:, 1]
        page = s["pages"][of, b // per].long()
        row = (b % per * B)[:, None] + torch.arange(B, device="cuda")
        s["M"][page, :, b % per] = s["K"][page[:, None], :, row].float().mean(1).to(dt)


def _cached(pool, s):
    """[seqs][hkv][max_len][d] in fp32, and which tokens are there"""
    t = torch.arange(s["max_len"], device="cuda")
    page = s["pages"][:, t // s["case"]["page"]].long()
    x = pool[page.clamp(min=0), :, (t % s["case"]["page"]).expand_as(page)]
    return x.transpose(1, 2).float(), page >= 0


def _softmax_rows(x, v, dt):
    """Rows of scores with -inf at what they do not see, values -> output, log of the sum"""
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = (x - m).exp()
    z = e.sum(-1, keepdim=True)
    y = torch.matmul(e, v) / torch.where(z > 0, z, 1.0)
    return y.to(dt), (m + z.log())[..., 0]


def _attend(s):
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    G, N, n = hq // hkv, s["max_new"], c["seqs"]
    K, there = _cached(s["K"], s)
    V, _ = _cached(s["V"], s)
    q = s["q"][s["row_at"]].float().reshape(n, N, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, G * N, d)
    x = torch.matmul(q, K.transpose(2, 3)).mul_(d ** -0.5).view(n, hkv, G, N, s["max_len"])
    at = s["seqs"][:, 0, None].long() + torch.arange(N, device="cuda")                    # [seqs][N]
    t = torch.arange(s["max_len"], device="cuda")
    seen = there[:, None] & (t <= at[..., None])
    if c["window"]:
        seen &= t > at[..., None] - c["window"]
    x.masked_fill_(~seen[:, None, None], -math.inf)
    y, lse = _softmax_rows(x.view(n, hkv, G * N, -1), V, _dt(c))
    y = y.view(n, hkv, G, N, d).permute(0, 3, 1, 2, 4).reshape(n, N, hq, d)
    lse = lse.view(n, hkv, G, N).permute(0, 3, 1, 2).reshape(n, N, hq)
    i = torch.arange(s["rows"], device="cuda") - s["seqs"][s["seq_of"], 2]
    s["out"].copy_(y[s["seq_of"], i])
    s["lse"].copy_(lse[s["seq_of"], i])


def _blocks(s):
    c = s["case"]
    hq, hkv, d, B, rows = c["hq"], c["hkv"], c["d"], c["block"], s["rows"]
    G, per = hq // hkv, c["page"] // B
    nb = -(-s["max_len"] // B)
    b = torch.arange(nb, device="cuda")
    page = s["pages"][:, b // per].long().clamp(min=0)
    M = s["M"][page, :, (b % per).expand_as(page)].transpose(1, 2).double()               # [seqs][hkv][nb][d]
    q = s["q"].view(rows, hkv, G, d)
    score = torch.matmul(M[s["seq_of"]], q.double().transpose(2, 3)).amax(-1)             # [rows][hkv][nb]
    have = (s["pos"] // B + 1)[:, None, None]                                             # blocks up to the token's own
    always = (b < have) & ((b < c["first"]) | (b >= have - c["last"]))
    score = score.masked_fill(always | (b >= have), -math.inf)
    best = score.sort(dim=-1, descending=True, stable=True)
    best = torch.where(best.values > -math.inf, best.indices, nb)[..., :c["top"]]
    taken = torch.zeros(rows, hkv, nb + 1, device="cuda", dtype=torch.bool).scatter_(2, best, True)[..., :nb] | always
    ids = torch.where(taken, b, nb).sort(-1).values[..., :min(nb, c["first"] + c["last"] + c["top"])]
    t = (ids[..., None] * B + torch.arange(B, device="cuda")).flatten(2)                  # [rows][hkv][tokens]
    seen = (t <= s["pos"][:, None, None]) & (ids < nb).repeat_interleave(B, -1)
    t = torch.where(seen, t, 0)
    page, row = s["pages"][s["seq_of"][:, None, None], t // c["page"]].long(), t % c["page"]
    head = torch.arange(hkv, device="cuda")[None, :, None]
    K, V = s["K"][page, head, row].float(), s["V"][page, head, row].float()               # [rows][hkv][tokens][d]
    x = torch.matmul(q.float(), K.transpose(2, 3)) * d ** -0.5
    y, _ = _softmax_rows(x.masked_fill(~seen[:, :, None], -math.inf), V, _dt(c))
    s["out"].copy_(y.reshape(rows, hq, d))


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------
def work(case):
    c = case
    hq, hkv, d, es, B = c["hq"], c["hkv"], c["d"], 2 if c["dtype"] == "bf16" else 4, c["block"]
    nbytes = flops = 0
    for n, m in _lengths(c):
        nbytes += 4 * -(-(n + m) // c["page"])                                            # page ids
        if c["op"] == "append":
            nbytes += 2 * m * (hq + 2 * hkv) * d * es
            flops += 3 * m * (hq + hkv) * c["rot"]
            if B:
                filled = (n + m) // B - n // B
                nbytes += hkv * d * es * (filled + (n % B if filled else 0))
                flops += filled * B * hkv * d
            continue
        nbytes += m * hq * d * 2 * es                                                     # queries and outputs
        if c["op"] == "attend":
            w = c["window"] or n + m
            seen = sum(min(w, n + i + 1) for i in range(m))
            nbytes += 2 * min(n + m, w + m - 1) * hkv * d * es + 4 * m * hq
            flops += 4 * hq * d * seen
        else:
            for i in range(m):
                have = (n + i) // B + 1
                kept = min(have, c["first"] + c["last"] + c["top"])
                tokens = kept * B - (have * B - (n + i + 1))
                flops += 4 * hq * d * tokens + (2 * hq * d * have if have > kept else 0)
                nbytes += 2 * tokens * hkv * d * es if i == 0 else 0                      # other tokens may take the same ones
            nbytes += (n + m) // B * hkv * d * es
    return {"bytes": nbytes, "flops": flops}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------------
def _rotate64(x, angle, c):
    """Every pair of channels as one complex number, turned by its angle."""
    r = c["rot"]
    pairs = x[..., :r].unflatten(-1, (r // 2, 2)) if c["adjacent"] else x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(angle), angle)[:, None]
    z = torch.view_as_real(z)
    return torch.cat([(z if c["adjacent"] else z.transpose(-1, -2)).flatten(-2), x[..., r:]], -1)


def _places(s, i, length):
    """(page, row) of the first `length` tokens of sequence i"""
    t = torch.arange(length, device="cuda")
    return s["pages"][i, t // s["case"]["page"]].long(), t % s["case"]["page"]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    hq, hkv, d, B = c["hq"], c["hkv"], c["d"], c["block"]
    G = hq // hkv
    if c["op"] == "append":
        out = {"q_rot": torch.empty(s["rows"], hq, d, device="cuda", dtype=torch.float64), "K": s["K"].double(), "V": s["V"].double()}
        if B:
            out["M"] = s["M"].double()
        for i, (n, m) in enumerate(_lengths(c)):
            r = slice(int(s["seqs"][i, 2]), int(s["seqs"][i, 2]) + m)
            angle = torch.arange(n, n + m, device="cuda", dtype=torch.float64)[:, None] * s["inv_freq"]
            out["q_rot"][r] = _rotate64(s["q"][r].double(), angle, c)
            page, row = _places(s, i, n + m)
            out["K"][page[n:], :, row[n:]] = _rotate64(s["k"][r].double(), angle, c)
            out["V"][page[n:], :, row[n:]] = s["v"][r].double()
            if B:
                a, e = n // B * B, (n + m) // B * B
                if e > a:
                    keys = out["K"][page[a:e], :, row[a:e]].unflatten(0, (-1, B))
                    out["M"][page[a:e:B], :, row[a:e:B] // B] = keys.mean(1)
        return out
    y = torch.zeros(s["rows"], hq, d, device="cuda", dtype=torch.float64)
    lse = torch.full((s["rows"], hq), -math.inf, device="cuda", dtype=torch.float64)
    for i, (n, m) in enumerate(_lengths(c)):
        page, row = _places(s, i, n + m)
        r0 = int(s["seqs"][i, 2])
        lo = max(0, n + 1 - c["window"]) if c["window"] else 0
        t = torch.arange(lo, n + m, device="cuda")
        for h in range(hkv):
            K, V = s["K"][page[lo:].clamp(min=0), h, row[lo:]].double(), s["V"][page[lo:].clamp(min=0), h, row[lo:]].double()
            if c["op"] == "blocks":
                blocks = torch.arange((n + m - 1) // B + 1, device="cuda")
                M = s["M"][page[::B], h, row[::B] // B].double()
            for j0 in range(0, m, 1024):
                j = torch.arange(j0, min(m, j0 + 1024), device="cuda")
                hidden = t > (n + j)[:, None]
                if c["window"]:
                    hidden |= t <= (n + j)[:, None] - c["window"]
                if c["op"] == "blocks":
                    for x in range(j.numel()):
                        have = (n + int(j[x])) // B + 1
                        taken = (blocks < c["first"]) | (blocks >= have - c["last"])
                        free = torch.nonzero(~taken[:have])[:, 0]
                        score = (M[free] @ s["q"][r0 + int(j[x]), h * G:h * G + G].double().T).amax(1)
                        taken[free[torch.argsort(-score, stable=True)[:c["top"]]]] = True
                        hidden[x] |= ~taken[t // B]
                for g in range(h * G, h * G + G):
                    x = (s["q"][r0 + j0:r0 + j0 + j.numel(), g].double() @ K.T) * d ** -0.5
                    x = x.masked_fill(hidden, -math.inf)
                    at = slice(r0 + j0, r0 + j0 + j.numel())
                    lse[at, g] = torch.logsumexp(x, 1)
                    y[at, g] = torch.softmax(x, 1) @ V
    return {"out": y, "lse": lse} if c["op"] == "attend" else {"out": y}
