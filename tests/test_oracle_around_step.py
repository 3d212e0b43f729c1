"""Oracle pins of the operators around a decode step: rotation, log probabilities, and
blocks shared, freed and moved (small cases worked out by hand, and bad arguments)."""
import numpy as np
import pytest

from oracle import logprobs as OL
from oracle import pages as OG
from oracle import rotate as OR


def test_rotation_turns_pairs_and_keeps_lengths():
    x = np.zeros((2, 1, 4))
    x[:, 0] = [1.0, 0.0, 0.0, 2.0]
    pos = np.array([0, 3])
    for adjacent, pairs in ((False, [(0, 2), (1, 3)]), (True, [(0, 1), (2, 3)])):
        out, _ = OR.norm_rope(x, pos, None, [0.5, 0.25], 0.0, 4, adjacent)
        assert np.array_equal(out[0], x[0])
        for (a, b), f in zip(pairs, (0.5, 0.25)):
            w = complex(x[1, 0, a], x[1, 0, b]) * np.exp(1j * 3 * f)
            assert np.allclose([out[1, 0, a], out[1, 0, b]], [w.real, w.imag], atol=1e-15)


def test_norm_before_rotation_and_dims_that_stay():
    rng = np.random.default_rng(0)
    x, g = rng.normal(size=(1, 2, 8)), rng.normal(size=8)
    out, size = OR.norm_rope(x, np.array([5]), g, [0.3, 0.1], 0.0, 4, False)
    y = x * g / np.sqrt((x ** 2).mean(-1, keepdims=True))
    assert np.allclose(out[..., 4:], y[..., 4:]) and (np.abs(out) <= size + 1e-12).all()
    assert np.allclose(out[..., 0] ** 2 + out[..., 2] ** 2, y[..., 0] ** 2 + y[..., 2] ** 2)


def test_positions():
    pos, bad = OR.positions(7, [0, 2, 2, 5], [10, 4, 0], 100)
    assert list(pos) == [10, 11, 0, 1, 2, -1, -1] and not bad
    pos, bad = OR.positions(3, None, [7, -1, 101], 100)
    assert list(pos) == [7, -1, -1] and bad


def test_logprobs_of_a_known_row():
    z = np.log([0.5, 0.25, 0.25])
    lp, h, ids, top = OL.token_logprobs(z, 2, 1.0, 2)
    assert np.isclose(lp, np.log(0.25)) and np.isclose(h, 1.5 * np.log(2))
    assert list(ids) == [0, 1] and np.allclose(top, np.log([0.5, 0.25]))
    lp, h, ids, top = OL.token_logprobs([0.0, -np.inf, 0.0], 1, 2.0, 3)
    assert lp == -np.inf and np.isclose(h, np.log(2)) and list(ids) == [0, 2, 1]
    assert np.isnan(OL.token_logprobs([0.0, 1.0], 2, 1.0, 0)[0])


@pytest.mark.parametrize("z", [[0.0, np.nan], [np.inf, 0.0], [-np.inf, -np.inf]], ids=["nan", "inf", "empty"])
def test_logprobs_of_rows_without_a_distribution(z):
    lp, h, ids, top = OL.token_logprobs(z, 0, 1.0, 2)
    assert np.isnan(lp) and np.isnan(h) and list(ids) == [-1, -1] and np.isnan(top).all()


def _pool(tables, ctx, P, shared=None):
    t = np.array(tables)
    return t, np.array(ctx), np.zeros(P, int) if shared is None else np.array(shared), np.arange(P) * 10.0


def test_fork_shares_full_blocks_and_copies_the_begun_one():
    t, ctx, sh, x = _pool([[3, 5, -1], [-1, -1, -1], [-1, -1, -1]], [20, 0, 0], 8)
    ids, free = np.array([6, 7, 1]), [0, 3]
    assert OG.fork([0, 0], [2, 1], t, ctx, sh, ids, free, 8, [x]) == 0
    assert t.tolist() == [[3, 5, -1], [3, 7, -1], [3, 6, -1]] and list(ctx) == [20, 20, 20]
    assert sh[3] == 2 and sh.sum() == 2 and free == [2, 3] and x[6] == x[7] == x[5] == 50.0


def test_fork_passes_over_bad_rows_and_stops_where_the_list_ends():
    t, ctx, sh, x = _pool([[0, 1], [-1, -1], [-1, -1], [2, -1]], [17, 0, 0, 16], 6)
    f = OG.fork([0, 0, 0, 3, 9], [1, 1, 0, 2, 2], t, ctx, sh, np.array([4]), [0, 1], 6, [x])
    assert f == OG.BAD_ROW and list(ctx) == [17, 17, 16, 16] and t[2].tolist() == [2, -1]
    t, ctx, sh, x = _pool([[0, 1], [-1, -1], [-1, -1], [-1, -1], [2, -1]], [17, 0, 0, 0, 16], 6)
    free = [0, 1]
    assert OG.fork([0, 0, 4], [1, 2, 3], t, ctx, sh, np.array([4]), free, 6, [x]) == OG.CACHE_FULL
    assert list(ctx) == [17, 17, 0, 0, 16] and free == [1, 1] and sh.tolist() == [1, 0, 0, 0, 0, 0]
    f = OG.fork([0], [2], t, ctx, sh, np.array([4]), [0, 2], 6, [x])
    assert f == OG.BAD_TABLE and ctx[2] == 0


def test_release_frees_what_nobody_holds():
    t, ctx, sh, _ = _pool([[3, 5], [3, 7], [3, 6]], [20, 20, 32], 8, [0, 0, 0, 2, 0, 0, 0, 0])
    ids, free = np.full(8, -1), [4, 4]
    assert OG.release([2, 0], t, ctx, sh, ids, free, 8) == 0
    assert list(ctx) == [0, 20, 0] and sh[3] == 0 and free == [2, 4] and list(ids[2:4]) == [5, 6]
    assert OG.release([1], t, ctx, sh, ids, free, 8) == 0
    assert free == [0, 4] and list(ids[:2]) == [3, 7]


def test_release_of_bad_rows_and_tables():
    t, ctx, sh, _ = _pool([[1, 1], [2, 9], [4, -1]], [32, 32, 999], 6)
    ids, free = np.full(4, -1), [1, 4]
    f = OG.release([0, 1, 0, 7, 2], t, ctx, sh, ids, free, 6)
    assert f == OG.BAD_ROW | OG.BAD_TABLE | OG.BAD_CTXLEN | OG.CACHE_FULL
    assert list(ctx) == [0, 0, 999] and free == [0, 4] and ids[0] == 2 and (sh == 0).all()
    assert OG.release([2], t, ctx, sh, ids, [0, 5], 6) == OG.BAD_TABLE


def test_compact_moves_used_blocks_down():
    t, ctx, sh, x = _pool([[7, 2], [7, 5], [-1, 4]], [32, 20, 0], 8, [0, 0, 0, 0, 0, 0, 0, 1])
    ids, free = np.full(8, -1), [3, 3]
    assert OG.compact(t, ctx, sh, ids, free, 8, [x]) == (0, 3)
    assert t.tolist() == [[1, 2], [1, 0], [-1, 4]] and sh.tolist() == [0, 1, 0, 0, 0, 0, 0, 0]
    assert x[1] == 70.0 and x[0] == 50.0 and free == [3, 8] and list(ids[3:]) == [3, 4, 5, 6, 7]
    t, ctx, sh, x = _pool([[9, 1]], [32], 4)
    assert OG.compact(t, ctx, None, np.zeros(4, int), [0, 0], 4, [x]) == (OG.BAD_TABLE, 1)
    assert t.tolist() == [[9, 0]]


def test_calls_reject_a_null_context():
    from paper_2603_03310_amd import ent
    lib = ent.load()
    prm = ent.make_qk_params(None, None, None, 1e-6, 0)
    assert lib.ent_qk_norm_rope(None, 1, 1, prm, None, 64, None, 64, None, None, None, 64, None, 64,
                                None) == ent.ENT_E_INVAL
    assert lib.ent_token_logprobs(None, 1, None, 0, 1, *[None] * 4, 0, None, None, None) == ent.ENT_E_INVAL
    assert lib.ent_cache_fork(None, 1, 1, *[None] * 6, 1, *[None] * 7) == ent.ENT_E_INVAL
    assert lib.ent_cache_release(None, 1, 1, *[None] * 5, 1, None, None) == ent.ENT_E_INVAL
    assert lib.ent_cache_compact(None, 1, *[None] * 4, 1, *[None] * 8) == ent.ENT_E_INVAL
