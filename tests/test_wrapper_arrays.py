"""Decoder.fork, release, compact, logprobs and rotate refuse arrays that the library would read or
write past their end, or take for another type; larger ones, as a program keeps them, do.  The
library itself is not called."""
import pytest
import torch

from paper_2603_03310_amd import ent
from paper_2603_03310_amd.runner import Decoder, make_config

P, R, MAXB, V, T = 40, 4, 5, 50, 6


@pytest.fixture
def dec(monkeypatch):
    d = Decoder.__new__(Decoder)
    d.cfg, d.ctx, d.calls = make_config(max_batch=8, num_q_heads=4, num_kv_heads=2, head_dim=64, max_blocks_per_seq=MAXB, num_pool_blocks=P, vocab=V), None, []
    for name in ("ent_cache_fork", "ent_cache_release", "ent_cache_compact", "ent_token_logprobs",
                 "ent_qk_norm_rope"):
        monkeypatch.setattr(ent, name, lambda *a, n=name: d.calls.append((n, a)))
    return d


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def pages(**kw):
    return dict(dict(src=ints(2), dst=ints(2), rows=ints(2), block_tables=ints(R, MAXB), ctx_lens=ints(R),
                     shared=ints(P), free_ids=ints(P), free_range=ints(2), n_used=ints(1)), **kw)


def call(dec, what, a):
    cache = dict(k_cache=None, v_cache=None, ksum=None)
    names = {"fork": ("src", "dst", "block_tables", "ctx_lens", "shared", "free_ids", "free_range"),
             "release": ("rows", "block_tables", "ctx_lens", "free_ids", "free_range", "shared"),
             "compact": ("block_tables", "ctx_lens", "free_ids", "free_range", "shared", "n_used")}[what]
    getattr(dec, what)(**{n: a[n] for n in names}, **({} if what == "release" else cache))


LONG = torch.int64
BAD = [("fork", "dst", ints(1)), ("fork", "dst", ints(3)), ("fork", "src", ints(2).to(LONG)),
       ("fork", "dst", ints(2).to(LONG)), ("fork", "dst", ints(4)[::2]),
       ("release", "rows", ints(2).to(LONG)), ("release", "rows", ints(4)[::2])]
for _w in ("fork", "release", "compact"):
    BAD += [(_w, "block_tables", ints(R - 1, MAXB)), (_w, "block_tables", ints(R, MAXB - 1)),
            (_w, "block_tables", ints(R, MAXB + 1)), (_w, "block_tables", ints(R, MAXB + 1)[:, :MAXB]),
            (_w, "block_tables", ints(R, MAXB).to(LONG)), (_w, "block_tables", ints(R * MAXB)),
            (_w, "ctx_lens", ints(R).to(LONG)), (_w, "ctx_lens", ints(R, 2)[:, 0]), (_w, "shared", ints(P - 1)),
            (_w, "shared", ints(P).to(LONG)), (_w, "free_ids", ints(P).to(LONG)), (_w, "free_ids", ints(2 * P)[::2]),
            (_w, "free_range", ints(1)), (_w, "free_range", ints(2).to(LONG))]
BAD += [("compact", "n_used", ints(0)), ("compact", "n_used", ints(1).to(LONG))]


@pytest.mark.parametrize("what,name,x", BAD, ids=lambda v: v if isinstance(v, str) else f"{tuple(v.shape)}{v.stride()}")
def test_block_calls_refuse(dec, what, name, x):
    with pytest.raises(ent.EntError) as e:
        call(dec, what, pages(**{name: x}))
    assert e.value.code == ent.ENT_E_INVAL and name in str(e.value) and not dec.calls


@pytest.mark.parametrize("what", ["fork", "release", "compact"])
def test_block_calls_pass_arrays_on(dec, what):
    call(dec, what, pages())
    call(dec, what, pages(block_tables=ints(R + 3, MAXB), shared=ints(P + 1), free_range=ints(3), free_ids=ints(P + 9),
                          n_used=ints(2)))
    call(dec, what, pages(src=ints(0), dst=ints(0), rows=ints(0), block_tables=ints(0, MAXB), ctx_lens=ints(0)))
    if what != "fork":
        call(dec, what, pages(shared=None, n_used=None))
    assert len(dec.calls) == (3 if what == "fork" else 4)
    n = {"fork": (2, 4), "release": (2, 4), "compact": (4,)}[what]
    assert all(c[1][1:1 + len(n)] == n for c in dec.calls[:2])


def rows(**kw):
    return dict(dict(logits=torch.zeros(T, V), tokens=ints(T), logprob=torch.zeros(T), entropy=torch.zeros(T),
                     top_ids=ints(T, 3), top_logprobs=torch.zeros(T, 3), temp=torch.ones(T)), **kw)


@pytest.mark.parametrize("name,x", [
    ("logits", torch.zeros(T, V - 1)), ("logits", torch.zeros(T, 2 * V)[:, :V - 1]), ("logits", torch.zeros(V)),
    ("logits", torch.zeros(T, V).double()), ("logits", torch.zeros(V, T).t()), ("tokens", ints(T).to(LONG)),
    ("tokens", ints(T - 1)), ("tokens", ints(2 * T)[::2]), ("logprob", torch.zeros(T - 1)),
    ("logprob", torch.zeros(T).double()), ("logprob", torch.zeros(2 * T)[::2]), ("entropy", torch.zeros(T - 1)),
    ("entropy", torch.zeros(T, dtype=torch.bfloat16)), ("temp", torch.zeros(T - 1)), ("temp", torch.zeros(T).double()),
    ("top_ids", ints(T - 1, 3)), ("top_ids", ints(T, 3).to(LONG)), ("top_ids", ints(T, 4)[:, :3]),
    ("top_logprobs", torch.zeros(T, 2)), ("top_logprobs", torch.zeros(T - 1, 3)),
    ("top_logprobs", torch.zeros(T, 3).double()), ("top_logprobs", torch.zeros(T, 4)[:, :3])],
    ids=lambda v: v if isinstance(v, str) else f"{tuple(v.shape)}{v.stride()}{v.dtype}")
def test_logprobs_refuse(dec, name, x):
    with pytest.raises(ent.EntError) as e:
        dec.logprobs(**rows(**{name: x}))
    assert e.value.code == ent.ENT_E_INVAL and name in str(e.value) and not dec.calls


def test_logprobs_pass_arrays_on(dec):
    dec.logprobs(**rows())
    dec.logprobs(**rows(logits=torch.zeros(T, V + 7, dtype=torch.bfloat16), tokens=ints(T + 2), logprob=torch.zeros(T + 1),
                        entropy=None, temp=torch.ones(T + 9), top_ids=ints(T + 1, 3), top_logprobs=torch.zeros(T + 4, 3)))
    dec.logprobs(**rows(tokens=None, logprob=None, temp=None, top_ids=None, top_logprobs=None))
    assert [c[1][1] for c in dec.calls] == [T] * 3 and dec.calls[1][1][4] == V + 7
    assert [c[1][9] for c in dec.calls] == [3, 3, 0]


def turned(starts=ints(4), ctx_lens=ints(3), gains=(torch.ones(64), torch.ones(64)), freq=torch.ones(16), B=3):
    q, k = torch.zeros(T, 4, 64), torch.zeros(T, 2, 64)
    return (B, ent.make_qk_params(*gains, freq, 1e-6, 32), q, k, q, k), dict(starts=starts, ctx_lens=ctx_lens)


@pytest.mark.parametrize("name,kw", [
    ("starts", dict(starts=ints(3))), ("starts", dict(starts=ints(4).to(LONG))), ("starts", dict(starts=ints(8)[::2])),
    ("ctx_lens", dict(ctx_lens=ints(2))), ("ctx_lens", dict(ctx_lens=ints(3).to(LONG))),
    ("q_gain", dict(gains=(torch.ones(63), None))), ("q_gain", dict(gains=(torch.ones(64).bfloat16(), None))),
    ("k_gain", dict(gains=(None, torch.ones(64).double()))), ("k_gain", dict(gains=(None, torch.ones(128)[::2]))),
    ("inv_freq", dict(freq=torch.ones(15))), ("inv_freq", dict(freq=torch.ones(16).double()))], ids=lambda v: v if isinstance(v, str) else "")
def test_rotate_refuses(dec, name, kw):
    a, b = turned(**kw)
    with pytest.raises(ent.EntError) as e:
        dec.rotate(*a, **b)
    assert e.value.code == ent.ENT_E_INVAL and name in str(e.value) and not dec.calls


def test_rotate_passes_arrays_on(dec):
    for kw in (dict(), dict(starts=ints(9), ctx_lens=ints(9)), dict(ctx_lens=None, gains=(None, None)),
               dict(starts=ints(1), B=0), dict(starts=None, B=3), dict(freq=torch.ones(40))):
        a, b = turned(**kw)
        dec.rotate(*a, **b)
    assert [c[1][1] for c in dec.calls] == [3, 3, 3, 0, 3, 3]
