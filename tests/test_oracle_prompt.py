"""Pins of the oracle's prompt operators against brute force, library routines
and closed forms."""
import numpy as np
import pytest

from oracle import prompt as OP


def test_plan_places_every_token_once():
    rng = np.random.default_rng(1)
    for _ in range(30):
        B, maxb = int(rng.integers(1, 6)), 6
        ctx = rng.integers(0, 40, B)
        n = rng.integers(0, 50, B)
        have = -(-ctx // 16)
        P = int(have.sum()) + 40
        ids = rng.permutation(P)
        tables = np.full((B, maxb), -1)
        at = 0
        for b in range(B):
            tables[b, :have[b]] = ids[at:at + have[b]]
            at += have[b]
        tab, starts, slots, lens, rngo, flags = OP.plan(n, ctx, tables, ids[at:], [0, len(ids) - at],
                                                        300, P)
        assert flags == 0 and list(np.diff(starts)) == list(n) and (lens == ctx + n).all()
        used = set()
        for b in range(B):
            for i in range(n[b]):
                pos = ctx[b] + i
                assert slots[starts[b] + i] == tab[b, pos // 16] * 16 + pos % 16
                used.add(int(slots[starts[b] + i]))
            assert (tab[b, -(-lens[b] // 16):] == -1).all()
        assert len(used) == n.sum() and (slots[starts[-1]:] == -1).all()
        assert rngo[0] == sum(-(-lens // 16) - have)


def test_plan_stops_at_the_first_misfit():
    tab, starts, slots, lens, r, flags = OP.plan([20, 40, 1], [0, 0, 0], np.full((3, 4), -1),
                                                 np.arange(10), [1, 5], 100, 10)
    assert list(starts) == [0, 20, 20, 20] and flags == OP.CACHE_FULL and list(r) == [3, 5]
    assert list(lens) == [20, 0, 0] and list(tab[0, :3]) == [1, 2, -1] and (tab[1:] == -1).all()


@pytest.mark.parametrize("G", [1, 4])
def test_attention_equals_torch_per_request(G):
    import torch
    rng = np.random.default_rng(2)
    starts, Hkv, d = [0, 3, 3, 4, 20], 2, 8
    q = rng.normal(size=(22, Hkv * G, d))
    k, v = rng.normal(size=(22, Hkv, d)), rng.normal(size=(22, Hkv, d))
    out, lse, mass, _ = OP.attention(q, k, v, starts, 0.3)
    for a, e in zip(starts[:-1], starts[1:]):
        if a == e:
            continue
        kk, vv = (np.repeat(x[a:e], G, 1).transpose(1, 0, 2) for x in (k, v))
        ref = torch.nn.functional.scaled_dot_product_attention(
            torch.tensor(q[a:e].transpose(1, 0, 2).copy()), torch.tensor(kk.copy()),
            torch.tensor(vv.copy()), is_causal=True, scale=0.3)
        assert np.abs(out[a:e] - ref.numpy().transpose(1, 0, 2)).max() < 1e-12
    assert np.isnan(out[20:]).all() and (mass[:20] >= np.abs(out[:20]) - 1e-15).all()
    assert np.allclose(lse[3], 0.3 * (q[3].reshape(Hkv, G, d) * k[3][:, None]).sum(2).ravel())


def test_e4m3_matches_torch():
    import torch
    vals = OP.e4m3_values()
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(vals, t, equal_nan=True)
    x = np.concatenate([np.random.default_rng(3).normal(size=4000) * 2.0 ** np.arange(-12, 8).repeat(200),
                        vals[np.isfinite(vals)], [448, 463.9, -1e9, np.inf, np.nan, 0.0]])
    ref = torch.tensor(x).clamp(-448, 448).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(OP.e4m3_round(x.astype(np.float32)), ref, equal_nan=True)


def test_scale_is_the_smallest_power_of_two():
    assert OP.scale8(np.array([448.0])) == 1.0 and OP.scale8(np.array([448.5])) == 2.0
    assert OP.scale8(np.array([0.0])) == 2.0 ** OP.MIN_EXP
    assert OP.scale8(np.array([np.inf, -3.0, np.nan])) == 2.0 ** -7


def test_store8_token_by_token_is_close_to_at_once():
    """Codes stay within one rounding of the value at the final scale, plus one per growth."""
    rng = np.random.default_rng(4)
    P, H, d, n = 2, 1, 4, 23
    x = rng.normal(size=(n, H, d)) * np.exp2(rng.integers(-3, 4, (n, 1, 1)))
    state = [np.zeros((P, H, 16, d)), np.zeros((P, H, d, 16)), np.ones((P, H)), np.ones((P, H)),
             np.zeros((P, H, d))]
    for t in range(n):
        OP.store8(*state, [t], x[t:t + 1], x[t:t + 1])
    back = (state[0] * state[2][:, :, None, None])[:, 0].reshape(32, d)[:n]
    top = (state[2] * OP.TOP).repeat(16)[:n, None]
    # Half a step relative (2^-4) twice, or half the smallest step (2^-10 of the scale).
    assert (np.abs(back - x[:, 0]) <= 2 * 2.0 ** -4 * np.abs(x[:, 0]) + top / 448 * 2.0 ** -9).all()
    assert np.allclose(state[4][0, 0], back[:16].mean(0)) and np.allclose(state[4][1, 0], back[16:].mean(0))


def test_store_equals_appends():
    from oracle import append as OA
    rng = np.random.default_rng(5)
    P, H, d, n = 3, 2, 4, 40
    k, v = rng.normal(size=(n, H, d)), rng.normal(size=(n, H, d))
    a, b = np.zeros((P, H, 16, d)), np.zeros((P, H, d, 16))
    c, e = a.copy(), b.copy()
    table = np.array([2, 0, 1])
    ks = np.zeros((P, H, d))
    OP.store(a, b, ks, [table[i // 16] * 16 + i % 16 for i in range(n)], k, v)
    for t in range(n):
        OA.append_token(c, e, table, t, k[t], v[t], 16)
    assert np.array_equal(a, c) and np.array_equal(b, e)
    assert np.allclose(ks[1], k[32:].mean(0))
