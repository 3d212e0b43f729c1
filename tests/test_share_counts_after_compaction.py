"""Share counts that a compaction leaves: the sequences that then hold each block, less one,
whatever the counts were before; none where nobody holds it.  Sequences that went without
ent_cache_release (a length set to 0, a row given to a fork, a length out of range) leave
counts that are too high: a block of theirs, handed out again, would never become free."""
import numpy as np
import pytest

from oracle import pages as OG
from oracle import prompt as OP
from tests.test_gpu_pages import Pool, decoder
from tests.test_gpu_parity import torch_cuda  # noqa: F401


def holders(tables, ctx, P):
    """Entries of all sequences that name each block, less one (0 at least)."""
    n = np.zeros(P, np.int64)
    for t, c in zip(tables, ctx):
        if 0 <= c <= tables.shape[1] * 16:
            for p in t[:-(-int(c) // 16)]:
                if 0 <= p < P:
                    n[p] += 1
    return np.maximum(n - 1, 0)


def new_lengths(p):
    p.d["ctx"].copy_(p.torch.tensor(p.ctx, dtype=p.torch.int32))


def test_the_oracle_frees_blocks_that_dropped_out():
    """Two sequences share block 7; both go by a length of 0, and 7 is handed out again."""
    P, tables = 8, np.array([[7, -1], [7, -1]])
    ctx, shared, ids, free = np.array([16, 16]), np.zeros(P, int), np.arange(P), [P, P]
    shared[7] = 1
    ctx[:] = 0
    assert OG.compact(tables, ctx, shared, ids, free, P) == (0, 0)
    assert (shared == 0).all() and free == [0, P]
    tables, _, _, lens, rng, _ = OP.plan([16 * 2, 16 * 2], ctx, tables, ids, free, 64, P)
    free = [int(x) for x in rng]
    tables, _, _, lens, rng, _ = OP.plan([0, 0], lens, tables, ids, free, 64, P)
    assert OG.release([0, 1], tables, np.array(lens), shared, ids, free, P) == 0 and free == [0, P]


def test_the_oracle_counts_who_is_left():
    tables = np.array([[3, 5], [3, 6], [3, 2], [9, 0]])
    ctx, shared = np.array([32, 20, 0, 999]), np.array([4, 1, 7, 2, 0, 0, 3, 1])
    ids, free = np.zeros(8, int), [0, 0]
    assert OG.compact(tables, ctx, shared, ids, free, 8) == (OG.BAD_CTXLEN, 3)
    # 3, 5 and 6 are in use: they move to 0, 1 and 2.
    assert tables[:2].tolist() == [[0, 1], [0, 2]] and shared.tolist() == [1, 0, 0, 0, 0, 0, 0, 0]


@pytest.mark.gpu
@pytest.mark.parametrize("kind,H,D", [("bf16", 2, 64), ("f32", 1, 64), ("q8", 3, 128)])
def test_sequences_that_went_without_a_release(torch_cuda, kind, H, D):
    """Lengths set to 0, rows given to another fork, lengths out of range: then every block that is
    handed out comes back."""
    lens = [0, 1, 15, 16, 17, 100, 256, 255, 33, 64, 64]
    p = Pool(torch_cuda, lens, 24, 200, 20, kind, H, D, seed=H)
    p.upload()
    with decoder(p) as dec:
        p.both(dec, "fork", [5, 5, 1, 6, 6, 6, 9, 9], [11, 12, 13, 14, 15, 16, 17, 18], flags=0)
        p.both(dec, "fork", [7, 10], [11, 17], flags=0)          # their rows, with what they hold
        for rows, n in (([6, 14, 15, 16], 0), ([9], -1), ([12], 0)):
            p.ctx[rows] = n
        new_lengths(p)
        p.both(dec, "compact", flags=OG.BAD_CTXLEN)
        assert np.array_equal(p.shared, holders(p.tables, p.ctx, p.P))
        p.ctx[9] = 0
        new_lengths(p)
        p.both(dec, "fork", [10, 17, 5], [6, 9, 12], flags=0)
        p.both(dec, "release", np.arange(24), flags=0)
        assert (p.shared == 0).all() and p.free == [0, 200] and sorted(p.ids) == list(range(200))


@pytest.mark.gpu
@pytest.mark.parametrize("fill", [-3, 5, "random"])
def test_counts_of_any_value(torch_cuda, fill):
    """Counts that nobody keeps; blocks listed by hundreds of rows, and twice in one; nothing moves
    in the second call."""
    rng = np.random.default_rng(3)
    lens = list(rng.integers(0, 400, 60)) + [16 * 300]
    P = sum(-(-n // 16) for n in lens) + 900
    p = Pool(torch_cuda, lens, 700, P, 302, "q8", 1, 64, seed=1)
    for r in range(61, 700):
        s = int(rng.integers(0, 61))
        p.tables[r], p.ctx[r] = p.tables[s], p.ctx[s] // 16 * 16
    p.tables[60, 5] = p.tables[60, 4]
    p.shared[:] = rng.integers(-9, 9, P) if fill == "random" else fill
    p.upload()
    with decoder(p) as dec:
        for _ in range(2):
            p.both(dec, "compact", flags=0)
            assert np.array_equal(p.shared, holders(p.tables, p.ctx, P)) and p.shared.max() > 5
            p.d["shared"].fill_(77)
            p.shared[:] = 77
        p.both(dec, "compact", shared=False, flags=0)
        assert (p.shared == 77).all()


@pytest.mark.gpu
def test_in_a_graph(torch_cuda):
    """A fork, a length of 0 and a compaction, replayed on the same state."""
    torch = torch_cuda
    p = Pool(torch, [100, 60, 16, 3], 8, 60, 8, seed=8)
    p.upload()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    src, dst = i32([0, 1, 0]), i32([4, 5, 6])
    with decoder(p) as dec:
        k, v, ksum, _ = p.caches()
        d = p.d

        def work():
            dec.fork(src, dst, d["tables"], d["ctx"], d["shared"], d["ids"], d["free"], k, v, ksum)
            d["ctx"][4:6].zero_()
            dec.compact(d["tables"], d["ctx"], d["ids"], d["free"], k, v, ksum, d["shared"], n_used=p.used)

        state = list(d.values()) + p.dp + [p.used]
        saved = [t.clone() for t in state]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=torch.cuda.Stream()):
            work()
        assert p.oracle("fork", [0, 1, 0], [4, 5, 6]) == 0
        p.ctx[4:6] = 0
        assert p.oracle("compact") == 0
        assert np.array_equal(p.shared, holders(p.tables, p.ctx, p.P))
        for _ in range(3):
            for t, x in zip(state, saved):
                t.copy_(x)
            g.replay()
            torch.cuda.synchronize()
            p.same()
            dec.compact(d["tables"], d["ctx"], d["ids"], d["free"], k, v, ksum, d["shared"])
            torch.cuda.synchronize()
            p.same()
        assert dec.device_status() == 0


@pytest.mark.gpu
def test_counts_in_another_array(torch_cuda):
    """Counts are written before tables and lengths are read again."""
    from paper_2603_03310_amd import ent
    p = Pool(torch_cuda, [20, 33], 4, 40, 4, seed=9)
    p.upload()
    d = p.d
    k, v, ksum, _ = p.caches()
    with decoder(p) as dec:
        for name in ("ctx", "tables", "ids"):
            with pytest.raises(ent.EntError) as e:
                ent.ent_cache_compact(dec.ctx, 4, d["tables"], d["ctx"], d[name], d["ids"], 40, d["free"], k, v, None,
                                      None, ksum)
            assert e.value.code == ent.ENT_E_INVAL and "aliases" in str(e.value), name
        torch_cuda.cuda.synchronize()
        p.same()
