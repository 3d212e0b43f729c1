"""The path of a request through the paged cache, as timed cases with a plain form.

A serving program gets prompts as packed rows (the tokens of all requests one behind the
other) and has the library find their place in the cache (ent_prompt_plan: block tables,
starts, slot map, from lengths on the GPU), write their keys and values there
(ent_prompt_store, ent_prompt_store_q8), attend over them causally (ent_prompt_attention),
and then decode.  With a cache held in 8 bits (e4m3, a scale per block and KV head) a decode
step reads it with ent_sparse_paged_decode_q8 and appends with ent_kv_append_q8.

`run` computes the same in elementary torch operations where `own` is false.  Head shapes and
lengths are those of the benchmark's workloads (an 8B-shaped step, a 70B-shaped loop, the fp32
`tiny` shape) and generic ones.  A case's lengths are a fixed set, dealt to the requests in an
order that the seed draws, so its work does not depend on the seed.

What a call updates in place and another call of the same kind would move on (the free list's
head, the context lengths of an append) has a copy of its own for each of SLOTS passes, so
every pass does the same work.
"""
from __future__ import annotations

import math

import torch

own = False

SLOTS = 4096
PAGE = 16                 # tokens per block
TOP = 448.0               # largest e4m3 value
MIN_EXP = -64             # smallest scale of an 8-bit tile: 2^-64
EXTRA = 64                # free blocks behind those that a plan needs

ATT = dict(kind="attention", q_heads=32, kv_heads=8, head_dim=128, dtype="bf16", fused=True,
           lse=False, spread="linear", empty=0)
DEC = dict(kind="decode8", q_heads=32, kv_heads=8, head_dim=128)


def listed():
    return [
        # Before a decode step every sequence of a batch gets room for one more token.
        dict(kind="plan", name="plan_growth", batch=64, lo=1, hi=1, ctx_lo=2048, ctx_hi=8192,
             room=0, spread="linear", empty=0),
        # Many new requests of very unequal lengths, rows padded past the last token.
        dict(kind="plan", name="plan_prompts", batch=256, lo=64, hi=32768, ctx_lo=0, ctx_hi=0,
             room=1000, spread="log", empty=0),
        # One interactive request's keys and values into a bf16 cache.
        dict(kind="store", name="store_request", batch=1, lo=2500, hi=2500, kv_heads=8,
             head_dim=128, dtype="bf16", cache="same", ctx_hi=0, spread="linear"),
        # A batch of prompts into an 8-bit cache; some continue requests that end inside a block.
        dict(kind="store", name="store_batch_8bit", batch=24, lo=301, hi=4001, kv_heads=8,
             head_dim=128, dtype="bf16", cache="q8", ctx_hi=40, spread="linear"),
        # Bring-up and debugging: fp32, small heads, as in the tiny workload.
        dict(ATT, name="attention_tiny_fp32", batch=4, q_heads=8, head_dim=64, dtype="f32",
             lo=128, hi=512, fused=False, lse=True),
        # One interactive request.
        dict(ATT, name="attention_request", batch=1, lo=2500, hi=2500),
        # A packed batch, ragged, down to single tokens and an empty request; the 70B head shape.
        dict(ATT, name="attention_packed", batch=24, q_heads=64, lo=1, hi=4001, spread="log",
             empty=1, lse=True),
        # A long document.
        dict(ATT, name="attention_document", batch=1, lo=32768, hi=32768),
        # One request's decode step.
        dict(DEC, name="decode8_request", batch=1, lo=2500, hi=2500, keep=0.5),
        # The 70B-shaped loop where the controller has settled: a sixth of the blocks kept.
        dict(DEC, name="decode8_loop", batch=128, q_heads=64, lo=4096, hi=16384, keep=0.17),
        # The new token of one request, and of a batch, into an 8-bit cache.
        dict(kind="append8", name="append8_request", batch=1, lo=2500, hi=2500, kv_heads=8,
             head_dim=128),
        dict(kind="append8", name="append8_batch", batch=128, lo=64, hi=2048, kv_heads=8,
             head_dim=128),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = [(32, 8, 128), (32, 8, 128), (64, 8, 128), (16, 4, 64), (10, 10, 128), (48, 6, 128),
         (16, 1, 64), (4, 2, 64)]


def draw(rng):
    kind = rng.choice(["plan", "store", "store", "attention", "attention", "attention", "decode8",
                       "decode8", "append8"])
    hq, hkv, d = rng.choice(HEADS)
    spread = rng.choice(["linear", "log"])
    if kind == "plan":
        batch = _between(rng, 1, 1024)
        hi = _between(rng, 1, max(2, min(32768, 800000 // batch)))
        return dict(kind="plan", batch=batch, lo=rng.randint(1, hi), hi=hi, ctx_lo=0,
                    ctx_hi=rng.choice([0, 0, _between(rng, 1, 8192)]), room=rng.choice([0, 17, 900]),
                    spread=spread, empty=rng.choice([0, 0, 5]))
    if kind == "store":
        batch = _between(rng, 1, 64)
        hi = _between(rng, 1, max(2, 50000 // batch))
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        return dict(kind="store", batch=batch, lo=rng.randint(1, hi), hi=hi, kv_heads=hkv, head_dim=d,
                    dtype=dtype, cache="same" if dtype == "f32" else rng.choice(["same", "q8"]),
                    ctx_hi=rng.choice([0, 40]), spread=spread)
    if kind == "attention":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        batch = _between(rng, 1, 64)
        # No more work than the long document's.
        hi = _between(rng, 1, max(2, int(min(24576, 32000 / math.sqrt(batch)))))
        if dtype == "f32":
            batch, hi = min(batch, 16), min(hi, 2048)
        if hq > 32:
            hi = min(hi, int(max(2, 20000 / math.sqrt(batch))))
        return dict(ATT, batch=batch, q_heads=hq, kv_heads=hkv, head_dim=d, dtype=dtype,
                    lo=rng.randint(1, hi), hi=hi, spread=spread, fused=rng.random() < 0.5,
                    lse=rng.random() < 0.5, empty=rng.choice([0, 0, 4]))
    batch = _between(rng, 1, 256)
    if kind == "append8":
        hi = _between(rng, 1, max(2, min(32768, 260000 // batch)))
        return dict(kind="append8", batch=batch, lo=rng.randint(1, hi), hi=hi, kv_heads=hkv,
                    head_dim=d)
    hi = _between(rng, 64, min(131072, 1200000 // batch))
    return dict(DEC, batch=batch, q_heads=hq, kv_heads=hkv, head_dim=d, lo=max(1, hi // 4), hi=hi,
                keep=rng.uniform(0.05, 0.18) if batch * hi > 600000 else rng.uniform(0.05, 0.75))


# --------------------------------------------------------------------------- inputs

def _spread(n, lo, hi, how):
    """n whole numbers over [lo, hi]: even steps, or even steps of the logarithm."""
    x = [(i + 0.5) / n for i in range(n)]
    if n == 1:
        return [hi]
    if how == "log":
        a, b = math.log(max(lo, 1)), math.log(max(hi, 1))
        return [min(hi, max(lo, int(round(math.exp(a + (b - a) * v))))) for v in x]
    return [int(round(lo + (hi - lo) * v)) for v in x]


def _lengths(c):
    """Lengths of the case's requests; one of every few empty where it says so."""
    v = _spread(c["batch"], c["lo"], c["hi"], c.get("spread", "linear"))
    if c.get("empty"):
        v[3::4 * c["empty"] + 7] = [0] * len(v[3::4 * c["empty"] + 7])
    return v


def _context(c):
    if not c.get("ctx_hi"):
        return [0] * c["batch"]
    return _spread(c["batch"], c.get("ctx_lo", 0), c["ctx_hi"], "linear")


def _deal(values, g):
    return [values[i] for i in torch.randperm(len(values), generator=g).tolist()]


def _pages(n):
    return -(-n // PAGE)


def _kept(c):
    """Kept blocks of each length."""
    return [min(_pages(n), max(4, math.ceil(c["keep"] * _pages(n)))) for n in _lengths(c)]


class _Inputs:
    """Everything that the seed draws, on the GPU."""


def _normal(shape, gd, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gd)


def _tiles8(shape, gd):
    """Codes and scales of an 8-bit cache: normal values, each tile with a range of its own."""
    codes = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
    scale = torch.empty(shape[:2], device="cuda")
    for a in range(0, shape[0], 16384):
        x = _normal((min(16384, shape[0] - a),) + tuple(shape[1:]), gd)
        x *= torch.exp(0.5 * _normal(x.shape[:2], gd))[:, :, None, None]
        s = torch.exp2(torch.ceil(torch.log2(x.abs().amax((2, 3)) / TOP)))
        codes[a:a + 16384] = (x / s[:, :, None, None]).clamp(-TOP, TOP).to(codes.dtype)
        scale[a:a + 16384] = s
    return codes, scale


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _tables(nbs, width, g):
    """Block tables of sequences of nbs blocks, in a pool that they fill in random order."""
    perm = torch.randperm(sum(nbs), generator=g).to(torch.int32)
    t = torch.full((len(nbs), width), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(nbs):
        t[b, :n] = perm[at:at + n]
        at += n
    return t


def _inputs(c, seed):
    x = _Inputs()
    g = torch.Generator()
    g.manual_seed(seed)
    gd = torch.Generator(device="cuda")
    gd.manual_seed(seed)
    B, kind = c["batch"], c["kind"]
    if kind in ("plan", "store"):
        x.lens, x.ctx = zip(*_deal(list(zip(_lengths(c), _context(c))), g))
        old = [_pages(n) for n in x.ctx]
        new = [_pages(n + m) for n, m in zip(x.ctx, x.lens)]
        need = sum(new) - sum(old)
        x.blocks = sum(new) + EXTRA
        x.total = sum(x.lens)
        x.width = max(1, max(new)) + 4
        x.tables = _tables(old, x.width, g).to("cuda")     # pool blocks 0 .. sum(old)
        ids = torch.randperm(need + EXTRA, generator=g).to(torch.int32) + sum(old)
        x.n_new, x.ctx_lens, x.ids = _i32(x.lens), _i32(x.ctx), ids.to("cuda")
        if kind == "plan":
            x.max_tokens = x.total + c["room"]
            return x
        H, d = c["kv_heads"], c["head_dim"]
        # Slots of the new tokens: what a plan of these requests gives.
        slots, at = [], 0
        for b in range(B):
            row = torch.cat([x.tables[b, :old[b]].cpu(), ids[at:at + new[b] - old[b]]]).long()
            at += new[b] - old[b]
            pos = torch.arange(x.ctx[b], x.ctx[b] + x.lens[b])
            slots.append(row[pos // PAGE] * PAGE + pos % PAGE)
        x.slots = torch.cat(slots).to("cuda")
        edt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        # Keys and values as one projection gives them, side by side; some tokens large.
        x.kv = _normal((x.total, 2, H, d), gd, edt)
        x.kv[::97] *= 8.0
        x.k, x.v = x.kv[:, 0], x.kv[:, 1]
        if c["cache"] == "q8":
            x.k_cache, x.k_scale = _tiles8((x.blocks, H, PAGE, d), gd)
            x.v_cache, x.v_scale = _tiles8((x.blocks, H, d, PAGE), gd)
        else:
            x.k_cache = _normal((x.blocks, H, PAGE, d), gd, edt)
            x.v_cache = _normal((x.blocks, H, d, PAGE), gd, edt)
        return x
    H, d = c["kv_heads"], c["head_dim"]
    x.lens = _deal(_lengths(c), g)
    if kind == "attention":
        x.total = sum(x.lens)
        edt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        starts = [0]
        for n in x.lens:
            starts.append(starts[-1] + n)
        x.starts = _i32(starts)
        Hq = c["q_heads"]
        if c["fused"]:           # views of one projection's rows
            rows = _normal((x.total, Hq + 2 * H, d), gd, edt)
            x.q, x.k, x.v = rows[:, :Hq], rows[:, Hq:Hq + H], rows[:, Hq + H:]
        else:
            x.q = _normal((x.total, Hq, d), gd, edt)
            x.k, x.v = _normal((x.total, H, d), gd, edt), _normal((x.total, H, d), gd, edt)
        return x
    grow = 1 if kind == "append8" else 0
    nbs = [_pages(n + grow) for n in x.lens]
    x.blocks, x.width = sum(nbs), max(nbs)
    x.rows = _tables(nbs, x.width, g)
    x.tables, x.ctx_lens = x.rows.to("cuda"), _i32(x.lens)
    x.k_cache, x.k_scale = _tiles8((x.blocks, H, PAGE, d), gd)
    x.v_cache, x.v_scale = _tiles8((x.blocks, H, d, PAGE), gd)
    if kind == "append8":
        x.k_new = _normal((B, H, d), gd, torch.bfloat16)
        x.v_new = _normal((B, H, d), gd, torch.bfloat16)
        x.k_new[::5] *= 16.0     # some past the range that their block has so far
        x.v_new[::7] *= 16.0
        return x
    x.q = _normal((B, c["q_heads"], d), gd, torch.bfloat16)
    keep = dict(zip(_lengths(c), _kept(c)))
    x.kept = torch.full((B, x.width), -1, dtype=torch.int32)
    x.nk = [keep[n] for n in x.lens]
    for b, n in enumerate(x.nk):                      # ascending, the last block among them
        some = torch.randperm(nbs[b] - 1, generator=g)[:n - 1]
        x.kept[b, :n] = torch.cat([some, torch.tensor([nbs[b] - 1])]).sort().values.to(torch.int32)
    x.kept, x.n_kept = x.kept.to("cuda"), _i32(x.nk)
    return x


# --------------------------------------------------------------------------- the calls

class _State:
    """A program's buffers; where the library runs, its context too."""

    ctx = None

    def __del__(self):
        if self.ctx:
            self.ent.ent_destroy(self.ctx)


def _handle(s, c, x):
    """The library context that a program keeps (its shapes are fixed there)."""
    from paper_2603_03310_amd import ent
    from paper_2603_03310_amd.runner import make_config

    s.ent = ent
    d, H = c.get("head_dim", 128), c.get("kv_heads", 8)
    s.ctx = ent.ent_init(make_config(
        max_batch=c["batch"], num_q_heads=c.get("q_heads", H), num_kv_heads=H, head_dim=d,
        max_blocks_per_seq=getattr(x, "width", 1), num_pool_blocks=getattr(x, "blocks", 1),
        kv_dtype=int(c.get("dtype", "bf16") == "bf16"), scale=1.0 / math.sqrt(d)))


def prepare(case, seed):
    c, x = case, _inputs(case, seed)
    s = _State()
    s.c, s.x, s.at = c, x, 0
    s.scale = 1.0 / math.sqrt(c.get("head_dim", 128))
    if own:
        _handle(s, c, x)
    s.stream = torch.cuda.current_stream().cuda_stream
    f32, i32 = dict(dtype=torch.float32, device="cuda"), dict(dtype=torch.int32, device="cuda")
    B = c["batch"]
    if c["kind"] == "plan":
        first = torch.tensor([0, x.ids.numel()], **i32)
        s.free = first.expand(SLOTS, 2).contiguous().unbind(0)
        s.starts, s.new_lens = torch.zeros(B + 1, **i32), torch.zeros(B, **i32)
        s.slots = torch.zeros(x.max_tokens, dtype=torch.int64, device="cuda")
    elif c["kind"] == "attention":
        s.out = torch.zeros((x.total, c["q_heads"], c["head_dim"]), dtype=x.q.dtype, device="cuda")
        s.lse = torch.zeros((x.total, c["q_heads"]), **f32) if c["lse"] else None
    elif c["kind"] == "decode8":
        s.out = torch.zeros((B, c["q_heads"], c["head_dim"]), **f32)
        s.lse = torch.zeros((B, c["q_heads"]), **f32)
    else:
        s.ksum = torch.zeros((x.blocks, c["kv_heads"], c["head_dim"]), **f32)
        if c["kind"] == "append8":
            s.lens = x.ctx_lens.expand(SLOTS, B).contiguous().unbind(0)
    return s


def run(s):
    i, c, x = s.at % SLOTS, s.c, s.x
    s.at += 1
    kind = c["kind"]
    if kind == "plan":
        free = s.free[i]
        if own:
            s.ent.ent_prompt_plan(s.ctx, c["batch"], x.n_new, x.ctx_lens, x.tables, x.ids,
                                  x.ids.numel(), free, x.max_tokens, s.starts, s.slots, s.new_lens,
                                  stream=s.stream)
        else:
            _plan(s, x, free)
        return dict(tables=x.tables, starts=s.starts, slots=s.slots, new_lens=s.new_lens,
                    free=free)
    if kind == "store":
        caches = dict(k_cache=x.k_cache, v_cache=x.v_cache, ksum=s.ksum)
        if c["cache"] == "q8":
            if own:
                s.ent.ent_prompt_store_q8(s.ctx, x.total, x.k, x.k.stride(0), x.v, x.v.stride(0),
                                          x.slots, x.k_cache, x.v_cache, x.k_scale, x.v_scale,
                                          s.ksum, stream=s.stream)
            else:
                _store8(s, x, x.slots, x.k, x.v)
            return dict(caches, k_scale=x.k_scale, v_scale=x.v_scale)
        if own:
            s.ent.ent_prompt_store(s.ctx, x.total, x.k, x.k.stride(0), x.v, x.v.stride(0), x.slots,
                                   x.k_cache, x.v_cache, s.ksum, stream=s.stream)
        else:
            _store(s, x)
        return caches
    if kind == "attention":
        if own:
            s.ent.ent_prompt_attention(s.ctx, c["batch"], x.total, x.q, x.q.stride(0), x.k,
                                       x.k.stride(0), x.v, x.v.stride(0), x.starts, s.out,
                                       s.out.stride(0), s.lse, stream=s.stream)
        else:
            _attention(s, x)
        return dict(out=s.out) if s.lse is None else dict(out=s.out, lse=s.lse)
    if kind == "decode8":
        if own:
            s.ent.ent_sparse_paged_decode_q8(s.ctx, c["batch"], x.q, x.k_cache, x.v_cache,
                                             x.k_scale, x.v_scale, x.tables, x.ctx_lens, x.kept,
                                             x.n_kept, s.out, s.lse, stream=s.stream)
        else:
            _decode8(s, x)
        return dict(out=s.out, lse=s.lse)
    lens = s.lens[i]
    if own:
        s.ent.ent_kv_append_q8(s.ctx, c["batch"], x.k_new, x.v_new, x.tables, lens, x.k_cache,
                               x.v_cache, x.k_scale, x.v_scale, s.ksum, stream=s.stream)
    else:
        at = lens.long()
        page = x.tables.gather(1, (at // PAGE)[:, None])[:, 0].long()
        _store8(s, x, page * PAGE + at % PAGE, x.k_new, x.v_new)
        lens += 1
    return dict(k_cache=x.k_cache, v_cache=x.v_cache, k_scale=x.k_scale, v_scale=x.v_scale,
                ksum=s.ksum, ctx_lens=lens)


# --------------------------------------------------------------------------- plain forms

def _plan(s, x, free):
    B, width = x.tables.shape
    n, ctx = x.n_new.long(), x.ctx_lens.long()
    have, want = (ctx + PAGE - 1) // PAGE, (ctx + n + PAGE - 1) // PAGE
    head, end = free[0].long(), free[1].long()
    blocks, tokens = torch.cumsum(want - have, 0), torch.cumsum(n, 0)
    fits = (blocks <= end - head) & (tokens <= x.max_tokens)    # in order: the first misfit ends it
    n, want = torch.where(fits, n, 0), torch.where(fits, want, have)
    ends, taken = torch.cumsum(n, 0), torch.cumsum(want - have, 0)
    s.starts[0] = 0
    s.starts[1:] = ends
    s.new_lens.copy_(ctx + n)
    j = torch.arange(width, device="cuda")
    at = (head + taken - (want - have))[:, None] + j[None, :] - have[:, None]
    fresh = (j[None, :] >= have[:, None]) & (j[None, :] < want[:, None])
    ids = x.ids[at.clamp(0, x.ids.numel() - 1)]
    x.tables.copy_(torch.where(fresh, ids, x.tables))
    t = torch.arange(x.max_tokens, device="cuda")
    b = torch.searchsorted(ends, t, right=True).clamp(max=B - 1)
    pos = ctx[b] + t - (ends - n)[b]
    page = x.tables[b, (pos // PAGE).clamp(max=width - 1)].long()
    s.slots.copy_(torch.where(t < ends[-1], page * PAGE + pos % PAGE, -1))
    free[0] += taken[-1].to(free.dtype)


def _groups(slots):
    """The blocks that the slots lie in, each slot's block among them, and what each has of slots."""
    page, inv = torch.unique(slots // PAGE, return_inverse=True)
    first = torch.full_like(page, PAGE).scatter_reduce(0, inv, slots % PAGE, "amin")
    last = torch.zeros_like(page).scatter_reduce(0, inv, slots % PAGE, "amax")
    return page, inv, first, last + 1


def _means(tiles, valid):
    """Mean key of each tile [n, H, 16, d] over its valid slots."""
    mask = torch.arange(PAGE, device="cuda")[None, :] < valid[:, None]
    kept = torch.where(mask[:, None, :, None], tiles, torch.zeros((), device="cuda"))
    return kept.sum(2) / valid[:, None, None]


def _store(s, x):
    page, slot = x.slots // PAGE, x.slots % PAGE
    x.k_cache[page, :, slot] = x.k
    x.v_cache[page, :, :, slot] = x.v
    blocks, _, _, valid = _groups(x.slots)
    s.ksum[blocks] = _means(x.k_cache[blocks].float(), valid)


def _scale8(top):
    """The smallest power of two, not under 2^MIN_EXP, times 448 that reaches `top`."""
    m, e = torch.frexp(top)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(top > 0, e, MIN_EXP).clamp(min=MIN_EXP)
    return torch.ldexp(torch.ones_like(top), e)


def _round8(v):
    return v.clamp(-TOP, TOP).to(torch.float8_e4m3fn).float()


def _merge8(old, scale, inv, row, first, new):
    """Tiles [n, H, 16, d] of values and their scales with the new rows in: a block that had tokens
    keeps its scale, or takes a larger one with its old values rounded again; others start anew."""
    n, H = old.shape[:2]
    amax = torch.zeros((n, H), device="cuda").scatter_reduce(
        0, inv[:, None].expand(-1, H), new.abs().amax(2), "amax")
    need = _scale8(amax)
    s = torch.where(first[:, None] > 0, torch.maximum(scale, need), need)
    slot = torch.arange(PAGE, device="cuda")
    again = ((s > scale) & (first[:, None] > 0))[:, :, None] & (slot[None, None, :] < first[:, None, None])
    codes = torch.where(again[..., None], _round8(old * (scale / s)[:, :, None, None]), old)
    codes[inv, :, row] = _round8(new / s[inv][:, :, None])
    return codes, s


def _codes(cache, at):
    """Some blocks of an 8-bit cache (indexed as bytes)."""
    return cache.view(torch.uint8)[at].view(cache.dtype).float()


def _put_codes(cache, at, codes):
    cache.view(torch.uint8)[at] = codes.contiguous().to(cache.dtype).view(torch.uint8)


def _store8(s, x, slots, k, v):
    blocks, inv, first, valid = _groups(slots)
    row = slots % PAGE
    codes, sc = _merge8(_codes(x.k_cache, blocks), x.k_scale[blocks], inv, row, first, k.float())
    _put_codes(x.k_cache, blocks, codes)
    x.k_scale[blocks] = sc
    s.ksum[blocks] = _means(codes, valid) * sc[:, :, None]
    codes, sc = _merge8(_codes(x.v_cache, blocks).transpose(2, 3), x.v_scale[blocks], inv, row,
                        first, v.float())
    _put_codes(x.v_cache, blocks, codes.transpose(2, 3))
    x.v_scale[blocks] = sc


def _attention(s, x):
    """One request after the other, as many of its queries at once as a gigabyte of scores holds."""
    Hq, d = x.q.shape[1:]
    H = x.k.shape[1]
    at = 0
    for n in x.lens:
        k = x.k[at:at + n].float().permute(1, 2, 0).contiguous()         # [H, d, n]
        v = x.v[at:at + n].float().transpose(0, 1).contiguous()          # [H, n, d]
        step = max(1, (1 << 28) // max(1, n * Hq))
        for a in range(0, n, step):
            m = min(step, n - a)
            u = a + m                                                    # keys up to the last query
            q = x.q[at + a:at + a + m].float().view(m, H, Hq // H, d)
            q = q.permute(1, 2, 0, 3).reshape(H, -1, d)                  # [H, G m, d]
            w = torch.matmul(q, k[:, :, :u]).view(H, -1, m, u) * s.scale
            late = torch.arange(u, device="cuda")[None, :] > torch.arange(a, u, device="cuda")[:, None]
            w.masked_fill_(late, -math.inf)
            top = w.amax(-1, keepdim=True)
            w = w.sub_(top).exp_()
            total = w.sum(-1, keepdim=True)
            o = torch.matmul(w.view(H, -1, u), v[:, :u]).view(H, -1, m, d) / total
            s.out[at + a:at + u] = o.permute(2, 0, 1, 3).reshape(m, Hq, d).to(s.out.dtype)
            if s.lse is not None:
                s.lse[at + a:at + u] = (top + torch.log(total))[..., 0].permute(2, 0, 1).reshape(m, Hq)
        at += n


def _decode8(s, x):
    B, Hq, d = x.q.shape
    H = x.k_cache.shape[1]
    most = max(x.nk)
    ids = x.kept[:, :most].long()
    page = x.tables.gather(1, ids.clamp(min=0)).long().clamp(min=0)      # [B, most]
    k = _codes(x.k_cache, page) * x.k_scale[page][..., None, None]       # [B, most, H, 16, d]
    k = k.permute(0, 2, 1, 3, 4).reshape(B, H, most * PAGE, d)
    q = x.q.float().view(B, H, Hq // H, d).transpose(2, 3).contiguous()
    w = torch.matmul(k, q) * s.scale                                     # [B, H, tokens, G]
    token = ids[:, :, None] * PAGE + torch.arange(PAGE, device="cuda")
    ok = (ids[:, :, None] >= 0) & (token < x.ctx_lens[:, None, None])
    w.masked_fill_(~ok.view(B, 1, -1, 1), -math.inf)
    top = w.amax(2, keepdim=True)
    w = w.sub_(top).exp_()
    total = w.sum(2, keepdim=True)
    del k
    v = _codes(x.v_cache, page) * x.v_scale[page][..., None, None]       # [B, most, H, d, 16]
    v = v.permute(0, 2, 3, 1, 4).reshape(B, H, d, most * PAGE)
    v.masked_fill_(~ok.view(B, 1, 1, -1), 0.0)
    o = torch.matmul(v, w) / total                                       # [B, H, d, G]
    s.out.copy_(o.transpose(2, 3).reshape(B, Hq, d))
    s.lse.copy_((top + torch.log(total)).view(B, Hq))


# --------------------------------------------------------------------------- what a pass needs

def work(case):
    c = case
    lens, kind = _lengths(c), c["kind"]
    if kind == "plan":
        blocks = sum(_pages(n + m) - _pages(n) for n, m in zip(_context(c), lens))
        return dict(bytes=16 * c["batch"] + 8 * blocks + 8 * (sum(lens) + c["room"]),
                    flops=4 * sum(lens))
    H, d = c["kv_heads"], c["head_dim"]
    e = 4 if c.get("dtype") == "f32" else 2
    if kind == "store":
        t = sum(lens)
        blocks = sum(_pages(n) for n in lens)
        out = 1 if c["cache"] == "q8" else e
        return dict(bytes=2 * t * H * d * (e + out) + 8 * t + blocks * H * d * 4,
                    flops=(5 if c["cache"] == "q8" else 1) * t * H * d)
    if kind == "attention":
        t, Hq = sum(lens), c["q_heads"]
        return dict(bytes=t * (2 * Hq + 2 * H) * d * e,
                    flops=2 * d * Hq * sum(n * (n + 1) for n in lens))
    if kind == "append8":
        # The block's keys are read for their mean, the new rows read and written.
        return dict(bytes=c["batch"] * H * d * (4 + 2 + 4) + sum(n % PAGE for n in lens) * H * d,
                    flops=sum(n % PAGE + 8 for n in lens) * H * d)
    kept = sum(_kept(c))
    Hq = c["q_heads"]
    return dict(bytes=kept * (2 * H * PAGE * d + 8 * H + 8) + c["batch"] * Hq * d * 6,
                flops=4 * kept * PAGE * Hq * d)


# --------------------------------------------------------------------------- 64 bits

def _e4m3(v):
    """The e4m3 value nearest to v, ties to the even one, at most 448 in size."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step).clamp(-TOP, TOP)


def _exact8(x, slots, k, v):
    """Caches, scales and summaries after new tokens at `slots`, block by block."""
    token = torch.full((x.blocks * PAGE,), -1, dtype=torch.int64, device="cuda")
    token[slots] = torch.arange(slots.numel(), device="cuda")
    token = token.view(-1, PAGE)
    at = torch.nonzero((token >= 0).any(1))[:, 0]
    token = token[at]
    fresh = token >= 0
    held = torch.cumsum(fresh.flip(1), 1).flip(1) > 0                     # up to the last new one
    grown = ~fresh[:, 0]
    r = {}
    for name, cache, scale, new in (("k", x.k_cache, x.k_scale, k), ("v", x.v_cache, x.v_scale, v)):
        old = _codes(cache, at).double()
        old = old.permute(0, 2, 1, 3) if name == "k" else old.permute(0, 3, 1, 2)     # [n, 16, H, d]
        rows = torch.where(fresh[:, :, None, None], new[token.clamp(min=0)].double(), 0.0)
        top = rows.abs().amax((1, 3))
        power = torch.ceil(torch.log2(top / TOP)).clamp(min=MIN_EXP, max=200.0)
        power = torch.where(TOP * torch.exp2(power) < top, power + 1, power)
        power = torch.where((TOP * torch.exp2(power - 1) >= top) & (power > MIN_EXP), power - 1, power)
        need, had = torch.exp2(power), scale[at].double()
        s = torch.where(grown[:, None] & (had > need), had, need)
        kept = torch.where((s > had)[:, None, :, None], _e4m3(old * (had / s)[:, None, :, None]), old)
        stale = ~held[:, :, None, None]
        kept = torch.where(stale, old, kept)
        codes = torch.where(fresh[:, :, None, None], _e4m3(rows / s[:, None, :, None]), kept)
        whole, scales = cache.double(), scale.double()
        whole[at] = codes.permute(0, 2, 1, 3) if name == "k" else codes.permute(0, 2, 3, 1)
        scales[at] = s
        r[name + "_cache"], r[name + "_scale"] = whole, scales
        if name == "k":
            mean = torch.where(stale, 0.0, codes).sum(1) / held.sum(1)[:, None, None]
            r["ksum"] = torch.zeros((x.blocks,) + tuple(mean.shape[1:]), dtype=torch.float64, device="cuda")
            r["ksum"][at] = mean * s[:, :, None]
    return r


def exact(case, seed):
    c, x = case, _inputs(case, seed)
    kind = c["kind"]
    if kind == "plan":
        return None                                   # whole numbers only
    f64 = dict(dtype=torch.float64, device="cuda")
    if kind == "attention":
        Hq, d, G = c["q_heads"], c["head_dim"], c["q_heads"] // c["kv_heads"]
        out, lse = torch.zeros((x.total, Hq, d), **f64), torch.zeros((x.total, Hq), **f64)
        first = 0
        for n in x.lens:
            for h in range(Hq if n else 0):
                k, v = (t[first:first + n, h // G].double().contiguous() for t in (x.k, x.v))
                for a in range(0, n, 4096):
                    b = min(n, a + 4096)
                    z = torch.mm(x.q[first + a:first + b, h].double(), k[:b].t().contiguous()) / math.sqrt(d)
                    z += torch.full((b - a, b), -math.inf, **f64).triu(a + 1)
                    p = torch.softmax(z, 1)
                    out[first + a:first + b, h] = torch.mm(p, v[:b])
                    lse[first + a:first + b, h] = torch.logsumexp(z, 1)
            first += n
        return dict(out=out, lse=lse) if c["lse"] else dict(out=out)
    H, d = c["kv_heads"], c["head_dim"]
    if kind == "decode8":
        Hq, G = c["q_heads"], c["q_heads"] // H
        out, lse = [], []
        for b, n in enumerate(x.lens):
            ids = x.kept[b, :x.nk[b]].long()
            page = x.tables[b, ids].long()
            rows = n - PAGE * int(ids[-1]) + PAGE * (x.nk[b] - 1)        # the last block is kept
            k = _codes(x.k_cache, page).double() * x.k_scale[page].double()[:, :, None, None]
            v = _codes(x.v_cache, page).double() * x.v_scale[page].double()[:, :, None, None]
            k = k.permute(1, 0, 2, 3).reshape(H, -1, d)[:, :rows].contiguous()
            v = v.permute(1, 0, 3, 2).reshape(H, -1, d)[:, :rows].contiguous()
            z = torch.matmul(x.q[b].double().view(H, G, d), k.transpose(1, 2).contiguous()) / math.sqrt(d)
            out.append(torch.matmul(torch.softmax(z, 2), v).reshape(Hq, d))
            lse.append(torch.logsumexp(z, 2).reshape(Hq))
        return dict(out=torch.stack(out), lse=torch.stack(lse))
    if kind == "append8":
        slots = torch.tensor([int(x.rows[b, n // PAGE]) * PAGE + n % PAGE for b, n in enumerate(x.lens)],
                             device="cuda")
        return dict(_exact8(x, slots, x.k_new, x.v_new), ctx_lens=None)
    if c["cache"] == "q8":
        return _exact8(x, x.slots, x.k, x.v)
    # Copies, and means over the tokens that a block holds afterwards.
    page, slot = x.slots // PAGE, x.slots % PAGE
    x.k_cache[page, :, slot] = x.k
    total, count = torch.zeros((x.blocks, H, d), **f64), torch.zeros(x.blocks, **f64)
    held = torch.zeros(x.blocks, dtype=torch.int64, device="cuda")
    held.index_reduce_(0, page, slot + 1, "amax")
    for i in range(PAGE):
        there = held > i
        total[there] += x.k_cache[there][:, :, i].double()
        count[there] += 1
    return dict(k_cache=None, v_cache=None, ksum=torch.where(count[:, None, None] > 0, total / count.clamp(min=1)[:, None, None],
                                       torch.zeros((), **f64)))
