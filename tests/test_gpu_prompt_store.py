"""ent_prompt_plan, ent_prompt_store and their 8-bit forms against the oracle:
tables, starts, slots and caches equal bit for bit; what a call is not to write
keeps a sentinel; device-side refusals raise their flags."""
import numpy as np
import pytest

from oracle import prompt as OP
from tests.prompt_data import config, to_dev
from tests.test_gpu_parity import torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu


def _i32(torch, x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda:0")


def _plan_case(rng, B, maxb, hi, ctx_hi):
    ctx = rng.integers(0, ctx_hi + 1, B)
    n = np.minimum(rng.integers(0, hi + 1, B), maxb * 16 - ctx)
    have = -(-ctx // 16)
    need = -(-(ctx + n) // 16) - have
    P = int(have.sum() + need.sum()) + 3
    ids = rng.permutation(P)
    tables = np.full((B, maxb), -1)
    at = 0
    for b in range(B):
        tables[b, :have[b]] = ids[at:at + have[b]]
        at += have[b]
    return ctx, n, tables, ids[at:], P


def _run_plan(torch, n, ctx, tables, ids, rng_, max_tokens, P, new_lens=True, **kw):
    from paper_2603_03310_amd.runner import Decoder
    B, maxb = tables.shape
    tab, free, starts = _i32(torch, tables), _i32(torch, rng_), _i32(torch, [-7] * (B + 2))
    slots = torch.full((max_tokens + 1,), -7, dtype=torch.int64, device="cuda:0")
    lens = _i32(torch, [-7] * (B + 1))
    with Decoder(**config(8, 8, 64, max_batch=max(B, 1), max_blocks_per_seq=maxb,
                          num_pool_blocks=P, **kw)) as dec:
        from paper_2603_03310_amd import ent
        idt = _i32(torch, ids)
        ent.ent_prompt_plan(dec.ctx, B, _i32(torch, n), _i32(torch, ctx), tab,
                            idt if len(ids) else None, len(ids), free, max_tokens, starts, slots,
                            lens if new_lens else None)
        torch.cuda.synchronize()
        flags = dec.device_status()
    starts, slots, lens = starts.cpu().numpy(), slots.cpu().numpy(), lens.cpu().numpy()
    assert starts[-1] == -7 and slots[-1] == -7 and lens[-1] == -7
    return tab.cpu().numpy(), starts[:-1], slots[:-1], lens[:-1], free.cpu().numpy(), flags


def _same_plan(got, want, new_lens=True):
    for name, a, b in zip(("tables", "starts", "slots", "lens", "free", "flags"), got, want):
        if name != "lens" or new_lens:
            assert np.array_equal(a, b), name
        else:
            assert (a == -7).all()


@pytest.mark.parametrize("B,maxb,hi,ctx_hi,room", [
    (1, 4, 0, 30, 0), (1, 4, 1, 60, 5), (3, 8, 40, 0, 0), (64, 40, 1, 600, 1), (65, 10, 100, 50, 300),
    (700, 6, 60, 30, 77), (2, 400, 6000, 17, 0), (1024, 3, 40, 5, 9)])
def test_plan(torch_cuda, B, maxb, hi, ctx_hi, room):
    rng = np.random.default_rng(B * 1000 + hi)
    ctx, n, tables, ids, P = _plan_case(rng, B, maxb, hi, ctx_hi)
    ids = np.concatenate([[0, 0], ids])                     # places before the head are not looked at
    want = OP.plan(n, ctx, tables, ids, [2, len(ids)], int(n.sum()) + room, P)
    assert want[5] == 0
    for new_lens in (True, False):
        _same_plan(_run_plan(torch_cuda, n, ctx, tables, ids, [2, len(ids)], int(n.sum()) + room, P,
                             new_lens), want, new_lens)


def test_plan_largest_batch(torch_cuda):
    rng = np.random.default_rng(7)
    ctx, n, tables, ids, P = _plan_case(rng, 4096, 4, 50, 10)
    want = OP.plan(n, ctx, tables, ids, [0, len(ids)], int(n.sum()), P)
    _same_plan(_run_plan(torch_cuda, n, ctx, tables, ids, [0, len(ids)], int(n.sum()), P,
                         num_q_heads=8, vocab=64), want)


@pytest.mark.parametrize("total", [524288, 524289, 700001])
def test_plan_many_tokens(torch_cuda, total):
    """Around the number of slots from which a workgroup takes more of them."""
    rng = np.random.default_rng(total)
    n = np.full(70, total // 70)
    n[33] = 0
    n[-1] += total - n.sum()
    ctx = rng.integers(0, 40, 70)
    maxb = int(np.max(-(-(ctx + n) // 16)))
    have, need = -(-ctx // 16), -(-(ctx + n) // 16) - -(-ctx // 16)
    P = int(have.sum() + need.sum())
    ids = rng.permutation(P)
    tables = np.full((70, maxb), -1)
    for b in range(70):
        tables[b, :have[b]] = ids[have[:b].sum():have[:b + 1].sum()]
    ids = ids[have.sum():]
    for rows in (total, total - 1):
        want = OP.plan(n, ctx, tables, ids, [0, len(ids)], rows, P)
        _same_plan(_run_plan(torch_cuda, n, ctx, tables, ids, [0, len(ids)], rows, P), want)


def test_plan_runs_out(torch_cuda):
    """Of blocks, of rows, of both; at the first request, at the last; no free list at all."""
    rng = np.random.default_rng(8)
    ctx, n, tables, ids, P = _plan_case(rng, 300, 8, 100, 20)
    total, need = int(n.sum()), len(ids)
    for blocks, rows in ((need // 2, total), (need, total // 3), (need - 4, total), (0, total),
                         (need, 0), (need // 3, total // 2), (1, 1)):
        want = OP.plan(n, ctx, tables, ids[:blocks], [0, blocks], rows, P)
        assert want[5] == OP.CACHE_FULL
        _same_plan(_run_plan(torch_cuda, n, ctx, tables, ids[:blocks], [0, blocks], rows, P), want)


def test_plan_bad_device_data(torch_cuda):
    """Requests out of range get nothing; free ids and table entries outside the pool give
    slot -1; a free range outside the list serves nobody."""
    from paper_2603_03310_amd import ent
    t = np.full((4, 4), -1)
    t[1, 0] = 99                                             # outside the pool of 12
    cases = [
        ([5, -3, 70, 9], [0, 0, 0, 0], t, list(range(8)), [0, 8],
         ent.ENT_DEV_BAD_CTXLEN | ent.ENT_DEV_CACHE_FULL),
        ([5, 4, 3, 9], [0, -1, 65, 0], t, list(range(8)), [0, 8], ent.ENT_DEV_BAD_CTXLEN),
        ([5, 20, 3, 9], [0, 7, 0, 0], t, list(range(8)), [0, 8], ent.ENT_DEV_BAD_TABLE),
        ([20, 2, 3, 9], [0, 0, 0, 0], t, [3, -4, 12, 5, 6, 7], [0, 6], ent.ENT_DEV_BAD_TABLE),
        ([5, 2, 3, 9], [0, 0, 0, 0], t, list(range(8)), [0, 9], None),
        ([5, 2, 3, 9], [0, 0, 0, 0], t, list(range(8)), [-1, 8], None),
        ([5, 2, 3, 9], [0, 0, 0, 0], t, list(range(8)), [6, 5], None),
    ]
    for n, ctx, tables, ids, r, flags in cases:
        want = OP.plan(n, ctx, tables, ids, r, 64, 12)
        got = _run_plan(torch_cuda, n, ctx, tables, ids, r, 64, 12)
        _same_plan(got[:5], want[:5])
        assert got[5] == (want[5] if flags is None else flags) == want[5]


def test_plan_grows_a_batch_again_and_again(torch_cuda):
    """The free list's head and the tables carry on from call to call, as before decode steps."""
    torch = torch_cuda
    from paper_2603_03310_amd.runner import Decoder
    rng = np.random.default_rng(9)
    ctx, _, tables, _, _ = _plan_case(rng, 20, 8, 0, 60)
    used = int((tables >= 0).sum())
    P = used + 60
    ids = used + rng.permutation(60)
    tab, free, lens = _i32(torch, tables), _i32(torch, [0, 60]), _i32(torch, ctx)
    starts, slots = _i32(torch, [0] * 21), torch.zeros(20, dtype=torch.int64, device="cuda:0")
    r = [0, 60]
    with Decoder(**config(8, 8, 64, max_blocks_per_seq=8, num_pool_blocks=P)) as dec:
        for _ in range(40):
            tables, st, sl, ctx, r, f = OP.plan([1] * 20, ctx, tables, ids, r, 20, P)
            dec.plan(20, _i32(torch, [1] * 20), lens, tab, _i32(torch, ids), free, starts, slots)
            lens += 1
            assert f == 0 and np.array_equal(slots.cpu().numpy(), sl)
        assert dec.device_status() == 0
    assert np.array_equal(tab.cpu().numpy(), tables) and np.array_equal(free.cpu().numpy(), r)


# --------------------------------------------------------------------------- stores

def _slots(rng, runs, P):
    """Slots of runs (first row, tokens) in blocks of their own; -1 for a run of first row -1."""
    free = list(rng.permutation(P))
    out = []
    for first, n in runs:
        if first < 0:
            out += [-1] * n
            continue
        pos = np.arange(first, first + n)
        blocks = [free.pop() for _ in range(pos[-1] // 16 + 1)]
        out += [blocks[x // 16] * 16 + x % 16 for x in pos]
    return np.array(out, np.int64)


RUNS = {
    "one": [(0, 1)],
    "last_row": [(15, 1)],
    "block": [(0, 16)],
    "middle": [(5, 7)],
    "over": [(13, 21)],
    "singles": [(i, 1) for i in range(16)] * 2,
    "mixed": [(0, 40), (-1, 3), (9, 7), (0, 1), (4, 60), (-1, 20), (15, 2), (0, 17), (0, 100)],
    "skips": [(-1, 50), (3, 3)],
}
STORE_HEADS = [(8, 128), (3, 64), (1, 128), (2, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("runs", RUNS.values(), ids=RUNS.keys())
@pytest.mark.parametrize("heads", STORE_HEADS, ids=str)
def test_store(torch_cuda, heads, runs, dtype):
    """Caches as the oracle's; the means as ent_block_summary's, bit for bit."""
    torch = torch_cuda
    from paper_2603_03310_amd import ent
    from paper_2603_03310_amd.runner import Decoder
    H, d = heads
    P = 48
    rng = np.random.default_rng(len(runs) + d)
    slots = _slots(rng, runs, P)
    T = len(slots)
    rows, val = to_dev(torch, rng.normal(size=(T, 2 * H + 1, d)), dtype)
    kc, kv = to_dev(torch, rng.normal(size=(P, H, 16, d)), dtype)
    vc, vv = to_dev(torch, rng.normal(size=(P, H, d, 16)), dtype)
    ksum = torch.full((P, H, d), -7.0, device="cuda:0")
    want = np.full((P, H, d), -7.0)
    OP.store(kv, vv, want, slots, val[:, 1:1 + H], val[:, 1 + H:])
    with Decoder(**config(H, H, d, dtype, num_pool_blocks=P)) as dec:
        dec.store(rows[:, 1:1 + H], rows[:, 1 + H:], torch.tensor(slots, device="cuda:0"), kc, vc, ksum)
        torch.cuda.synchronize()
        assert dec.device_status() == 0
        assert np.array_equal(kc.double().cpu().numpy(), kv)
        assert np.array_equal(vc.double().cpu().numpy(), vv)
        got = ksum.cpu().numpy()
        # A float32 sum of up to 16 values and a division: 16 half steps of their magnitude.
        assert np.abs(got - want).max() <= 17 * 2.0 ** -24 * np.abs(kv).max()
        # The same blocks as sequences of one block each, through ent_block_summary.
        hit = np.unique(slots[slots >= 0] // 16)
        ln = [int((slots[slots // 16 == p] % 16).max()) + 1 for p in hit]
        again = torch.full_like(ksum, -7.0)
        tab = torch.full((len(hit), 64), -1, dtype=torch.int32, device="cuda:0")
        tab[:, 0] = _i32(torch, hit)
        ent.ent_block_summary(dec.ctx, len(hit), kc, tab, _i32(torch, ln), again)
        assert torch.equal(again, ksum)


def _codes(torch, rng, shape):
    """Codes of any finite value, and the values."""
    c = rng.integers(0, 256, shape).astype(np.uint8)
    c = np.where((c & 0x7f) == 0x7f, 0x31, c).astype(np.uint8)
    return torch.tensor(c, device="cuda:0"), OP.e4m3_values()[c]


@pytest.mark.parametrize("pow2", [True, False], ids=["pow2", "any_scale"])
@pytest.mark.parametrize("runs", RUNS.values(), ids=RUNS.keys())
@pytest.mark.parametrize("heads", STORE_HEADS, ids=str)
def test_store_q8(torch_cuda, heads, runs, pow2):
    """Codes and scales equal the oracle's, where blocks begin, go on, and outgrow their scale."""
    torch = torch_cuda
    from paper_2603_03310_amd.runner import Decoder
    H, d = heads
    P = 48
    rng = np.random.default_rng(len(runs) + d + 1)
    slots = _slots(rng, runs, P)
    T = len(slots)
    x = rng.normal(size=(T, 2, H, d)) * np.exp2(rng.integers(-6, 7, (T, 2, H, 1)))
    x[rng.random(T) < 0.1] = 0.0
    rows, val = to_dev(torch, x)
    kc, kv = _codes(torch, rng, (P, H, 16, d))
    vc, vv = _codes(torch, rng, (P, H, d, 16))
    ks, vs = (np.exp2(rng.integers(-9, -2, (P, H))).astype(np.float32) for _ in range(2))
    if not pow2:
        ks, vs = (s * rng.uniform(1, 2, (P, H)).astype(np.float32) for s in (ks, vs))
    dks, dvs = torch.tensor(ks, device="cuda:0"), torch.tensor(vs, device="cuda:0")
    ksum = torch.full((P, H, d), -7.0, device="cuda:0")
    want = np.full((P, H, d), -7.0)
    OP.store8(kv, vv, ks, vs, want, slots, val[:, 0], val[:, 1])
    with Decoder(**config(H, H, d, num_pool_blocks=P)) as dec:
        dec.store(rows[:, 0], rows[:, 1], torch.tensor(slots, device="cuda:0"), kc, vc, ksum, dks, dvs)
        torch.cuda.synchronize()
        assert dec.device_status() == 0
    table = OP.e4m3_values()
    assert np.array_equal(dks.cpu().numpy(), ks) and np.array_equal(dvs.cpu().numpy(), vs)
    assert np.array_equal(table[kc.cpu().numpy()], kv)
    assert np.array_equal(table[vc.cpu().numpy()], vv)
    # An exact sum, a division and a product: two half steps (and a step's slack).
    assert np.allclose(ksum.cpu().numpy(), want, rtol=2.0 ** -22, atol=0)


def test_store_q8_not_finite_and_tiny(torch_cuda):
    """Infinities saturate at the range of the finite values, NaN stay; zeros and values
    under the smallest scale."""
    torch = torch_cuda
    from paper_2603_03310_amd.runner import Decoder
    x = np.zeros((48, 1, 64))
    x[:16] = np.random.default_rng(1).normal(size=(16, 1, 64))
    x[3, 0, 5], x[4, 0, 6], x[5, 0, 7] = np.inf, -np.inf, np.nan
    x[32:] = 2.0 ** -70
    rows, val = to_dev(torch, x)
    kc = torch.zeros(3, 1, 16, 64, dtype=torch.uint8, device="cuda:0")
    vc = torch.zeros(3, 1, 64, 16, dtype=torch.uint8, device="cuda:0")
    ks, vs = torch.zeros(3, 1, device="cuda:0"), torch.zeros(3, 1, device="cuda:0")
    ksum = torch.zeros(3, 1, 64, device="cuda:0")
    kv, vv = np.zeros((3, 1, 16, 64)), np.zeros((3, 1, 64, 16))
    wk, wv = np.zeros((3, 1), np.float32), np.zeros((3, 1), np.float32)
    with Decoder(**config(1, 1, 64, num_pool_blocks=3)) as dec:
        dec.store(rows, rows, torch.arange(48, device="cuda:0"), kc, vc, ksum, ks, vs)
        torch.cuda.synchronize()
    OP.store8(kv, vv, wk, wv, np.zeros((3, 1, 64)), np.arange(48), val, val)
    table = OP.e4m3_values()
    assert np.array_equal(table[kc.cpu().numpy()], kv, equal_nan=True)
    assert np.array_equal(table[vc.cpu().numpy()], vv, equal_nan=True)
    assert np.array_equal(ks.cpu().numpy(), wk) and wk[1, 0] == 2.0 ** -64
    assert kv[0, 0, 3, 5] == 448 and kv[0, 0, 4, 6] == -448 and np.isnan(kv[0, 0, 5, 7])


def test_store_slots_outside_the_pool(torch_cuda):
    torch = torch_cuda
    from paper_2603_03310_amd import ent
    from paper_2603_03310_amd.runner import Decoder
    x = torch.ones(20, 2, 64, dtype=torch.bfloat16, device="cuda:0")
    kc = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device="cuda:0")
    vc, ksum = torch.zeros(4, 2, 64, 16, dtype=torch.bfloat16, device="cuda:0"), torch.zeros(4, 2, 64, device="cuda:0")
    for far in (64, -2, 1 << 40, -(1 << 40)):
        slots = torch.arange(20, device="cuda:0")
        slots[18:] = far
        kc.zero_()
        with Decoder(**config(2, 2, 64, num_pool_blocks=4)) as dec:
            dec.store(x, x, slots, kc, vc, ksum)
            assert dec.device_status() == ent.ENT_DEV_BAD_TABLE
        assert (kc[0] == 1).all() and (kc[1, :, :2] == 1).all() and (kc[1, :, 2:] == 0).all()
        assert (kc[2:] == 0).all()


def test_refusals(torch_cuda):
    torch = torch_cuda
    from paper_2603_03310_amd import ent
    from paper_2603_03310_amd.runner import Decoder
    x = torch.zeros(16, 2, 64, dtype=torch.bfloat16, device="cuda:0")
    kc = torch.full((4, 2, 16, 64), -7.0, dtype=torch.bfloat16, device="cuda:0")
    slots, ksum = torch.arange(16, device="cuda:0"), torch.zeros(4, 2, 64, device="cuda:0")
    sc = torch.ones(4, 2, device="cuda:0")
    i = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda:0")
    n_new, ctx, tab, ids, rng, starts = i(2), i(2), i(128), i(4), i(2), i(3)
    I, U = ent.ENT_E_INVAL, ent.ENT_E_UNSUPPORTED

    def refuse(f, good, bads):
        for bad, code in bads:
            with pytest.raises(ent.EntError) as e:
                f(**{**good, **bad})
            assert e.value.code == code and str(e.value), bad

    with Decoder(**config(2, 2, 64, max_batch=2, num_pool_blocks=4)) as dec:
        refuse(lambda **k: ent.ent_prompt_plan(dec.ctx, **k),
               dict(B=2, n_new=n_new, ctx_lens=ctx, block_tables=tab, free_ids=ids, n_ids=4,
                    free_range=rng, max_tokens=16, starts=starts, slots=slots),
               [(dict(B=3), I), (dict(B=-1), I), (dict(n_ids=-1), I), (dict(max_tokens=-1), I),
                (dict(max_tokens=ent.ENT_MAX_PACKED_TOKENS + 1), U), (dict(n_new=None), I),
                (dict(ctx_lens=None), I), (dict(block_tables=None), I), (dict(free_ids=None), I),
                (dict(free_range=None), I), (dict(starts=None), I), (dict(slots=None), I),
                (dict(new_lens=ctx), I), (dict(new_lens=n_new), I), (dict(starts=ctx), I), (dict(starts=n_new), I),
                (dict(slots=slots.data_ptr() + 4), I)])
        common = [(dict(T=-1), I), (dict(T=ent.ENT_MAX_PACKED_TOKENS + 1), U), (dict(k=None), I),
                  (dict(v=None), I), (dict(slots=None), I), (dict(k_cache=None), I),
                  (dict(v_cache=None), I), (dict(ksum=None), I), (dict(ldk=127), I),
                  (dict(ldk=132), I), (dict(ldv=64), I), (dict(k=x.data_ptr() + 8), I),
                  (dict(k_cache=kc.data_ptr() + 8), I)]
        good = dict(T=16, k=x, ldk=128, v=x, ldv=128, slots=slots, k_cache=kc, v_cache=kc, ksum=ksum)
        good8 = dict(good, k_scale=sc, v_scale=sc)
        refuse(lambda **k: ent.ent_prompt_store(dec.ctx, **k), good, common)
        refuse(lambda **k: ent.ent_prompt_store_q8(dec.ctx, **k), good8,
               common + [(dict(k_scale=None), I), (dict(v_scale=None), I),
                         (dict(ksum=ksum.data_ptr() + 4), I)])
        app = dict(B=2, k_new=x, v_new=x, block_tables=tab, ctx_lens=ctx, k_cache=kc, v_cache=kc,
                   k_scale=sc, v_scale=sc, ksum=ksum)
        refuse(lambda **k: ent.ent_kv_append_q8(dec.ctx, **k), app,
               [(dict(B=3), I), (dict(B=-1), I), (dict(k_new=x.data_ptr() + 2), I),
                (dict(ksum=ksum.data_ptr() + 8), I)] +
               [({f: None}, I) for f in app if f != "B"])
        dcd = dict(B=2, q=x, k_cache=kc, v_cache=kc, k_scale=sc, v_scale=sc, block_tables=tab,
                   ctx_lens=ctx, kept=tab, n_kept=ctx, out=ksum)
        refuse(lambda **k: ent.ent_sparse_paged_decode_q8(dec.ctx, **k), dcd,
               [(dict(B=3), I), (dict(B=-1), I), (dict(out=ksum.data_ptr() + 4), I)] +
               [({f: None}, I) for f in dcd if f != "B"])
        # Nothing to do: nothing needed.
        ent.ent_prompt_plan(dec.ctx, 0, None, None, None, None, 0, None, 0, None, None)
        ent.ent_prompt_store(dec.ctx, 0, None, 0, None, 0, None, None, None, None)
        ent.ent_prompt_store_q8(dec.ctx, 0, None, 0, None, 0, None, None, None, None, None, None)
        ent.ent_kv_append_q8(dec.ctx, 0, None, None, None, None, None, None, None, None, None)
        ent.ent_sparse_paged_decode_q8(dec.ctx, 0, *([None] * 10))
        torch.cuda.synchronize()
        assert (kc == -7).all() and dec.device_status() == 0
    # An 8-bit cache: bf16 contexts with mean-key scoring only.
    for kw in (dict(kv_dtype=ent.ENT_F32), dict(scoring=ent.ENT_SCORE_EXACT)):
        with Decoder(**config(2, 2, 64, max_batch=2, num_pool_blocks=4, **kw)) as dec:
            for f, g in ((ent.ent_prompt_store_q8, good8), (ent.ent_kv_append_q8, app),
                         (ent.ent_sparse_paged_decode_q8, dcd)):
                with pytest.raises(ent.EntError) as e:
                    f(dec.ctx, **g)
                assert e.value.code == U
    # The exact mode keeps no summaries: the store needs none.
    with Decoder(**config(2, 2, 64, num_pool_blocks=4, scoring=ent.ENT_SCORE_EXACT)) as dec:
        ent.ent_prompt_store(dec.ctx, **{**good, "ksum": None, "v_cache": kc.clone()})
        torch.cuda.synchronize()
    assert (kc[0] == 0).all() and (kc[1:] == -7).all()
