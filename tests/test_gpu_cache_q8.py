"""The 8-bit cache in decoding: ent_sparse_paged_decode_q8 against the float64
oracle, ent_kv_append_q8 against ent_prompt_store_q8 and the oracle, and both
captured in a graph."""
import numpy as np
import pytest

from oracle import attention as OA
from oracle import prompt as OP
from tests.prompt_data import U32, config, host, to_dev
from tests.test_gpu_parity import torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

HEADS = [(32, 8, 128), (8, 8, 64), (16, 1, 128), (4, 2, 64), (12, 3, 128), (128, 8, 128), (64, 32, 64)]


def _i32(torch, x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda:0")


def _cache(torch, rng, P, H, d, pow2):
    """Codes of unit-like values, anything in slots that hold no token (the caller says which)."""
    out = []
    for shape in ((P, H, 16, d), (P, H, d, 16)):
        x = np.clip(rng.normal(size=shape) * 60, -448, 448)
        t = torch.tensor(x, device="cuda:0").float().to(torch.float8_e4m3fn).view(torch.uint8)
        s = np.exp2(rng.integers(-8, -4, (P, H))).astype(np.float32)
        if not pow2:
            s = (s * rng.uniform(1, 2, (P, H))).astype(np.float32)
        out += [t, torch.tensor(s, device="cuda:0")]
    return out


def _decode(torch, lens, keep, heads, seed=0, pow2=True, spoil=True, maxb=64, scale=None):
    """Runs the decode over keep[b] random kept blocks of each sequence (None: all)."""
    from paper_2603_03310_amd.runner import Decoder
    from paper_2603_03310_amd import ent
    Hq, H, d = heads
    rng = np.random.default_rng(seed)
    B = len(lens)
    nbs = [-(-n // 16) for n in lens]
    P = max(1, sum(nbs)) + 2
    perm = rng.permutation(P)
    tab = np.full((B, maxb), -1)
    at = 0
    for b, nb in enumerate(nbs):
        tab[b, :nb] = perm[at:at + nb]
        at += nb
    kc, ks, vc, vs = _cache(torch, rng, P, H, d, pow2)
    if spoil:            # codes past each sequence's end: NaN
        for b, n in enumerate(lens):
            if n % 16:
                kc[tab[b, n // 16], :, n % 16:] = 0x7f
                vc[tab[b, n // 16], :, :, n % 16:] = 0xff
    kept = np.full((B, maxb), -1)
    nk = []
    for b, nb in enumerate(nbs):
        k = nb if keep is None else min(nb, keep[b])
        nk.append(k)
        kept[b, :k] = np.sort(rng.choice(nb, k, replace=False)) if k else []
    q, qv = to_dev(torch, rng.normal(size=(B, Hq, d)))
    out = torch.full((B, Hq, d), -7.0, device="cuda:0")
    lse = torch.full((B, Hq), -7.0, device="cuda:0")
    cfg = config(Hq, H, d, max_batch=B, max_blocks_per_seq=maxb, num_pool_blocks=P)
    if scale is not None:
        cfg["scale"] = scale
    with Decoder(**cfg) as dec:
        ent.ent_sparse_paged_decode_q8(dec.ctx, B, q, kc, vc, ks, vs, _i32(torch, tab), _i32(torch, lens),
                                       _i32(torch, kept), _i32(torch, nk), out, lse)
        torch.cuda.synchronize()
        assert dec.device_status() == 0
    table = OP.e4m3_values()
    K = table[kc.cpu().numpy()] * host(ks)[:, :, None, None]
    V = table[vc.cpu().numpy()] * host(vs)[:, :, None, None]
    o, l = host(out), host(lse)
    sc = float(np.float32(cfg["scale"]))
    for b, n in enumerate(lens):
        Kb = K[tab[b, :nbs[b]]].transpose(0, 2, 1, 3).reshape(-1, H, d)[:n]
        Vb = V[tab[b, :nbs[b]]].transpose(0, 3, 1, 2).reshape(-1, H, d)[:n]
        ref, rl = OA.sparse_decode(qv[b], Kb, Vb, kept[b, :nk[b]], 16, sc)
        mass, _ = OA.sparse_decode(qv[b], Kb, np.abs(Vb), kept[b, :nk[b]], 16, sc)
        if nk[b] == 0:
            assert (o[b] == 0).all() and np.isneginf(l[b]).all()
            continue
        span = abs(sc) * np.max(np.sum(np.abs(qv[b])[:, None] * np.abs(np.repeat(Kb, Hq // H, 1)
                                                                     .transpose(1, 0, 2)), 2), 1)
        # Exact products (codes and queries have 4 and 8 bits), so a score is off by its sum's
        # rounding and by two products with its scale; weights of 24 bits, split exactly but
        # for 2^-24; sums over n tokens.
        ds = 2 * (d + 8) * U32 * span + 2.0 ** -20
        bound = (ds[:, None] + (4 * n + 8) * U32) * mass
        assert not np.isnan(o[b]).any()
        assert (np.abs(o[b] - ref) <= bound).all(), (b, n, np.abs((o[b] - ref) / bound).max())
        assert (np.abs(l[b] - rl) <= ds + 2 * n * U32 + 4 * U32 * np.abs(rl)).all()


@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_all_blocks(torch_cuda, heads):
    _decode(torch_cuda, [1, 15, 16, 17, 63, 64, 65, 333, 1000], None, heads)


@pytest.mark.parametrize("heads", HEADS[:4], ids=str)
def test_kept_blocks_and_any_scale(torch_cuda, heads):
    _decode(torch_cuda, [500, 0, 77, 1000, 16, 640], [3, 0, 5, 0, 1, 22], heads, seed=2, pow2=False)


def test_one_long_sequence_and_a_large_batch(torch_cuda):
    _decode(torch_cuda, [20011], None, (16, 4, 64), seed=3, maxb=1300)
    rng = np.random.default_rng(4)
    lens = rng.integers(0, 400, 200).tolist()
    _decode(torch_cuda, lens, rng.integers(0, 26, 200).tolist(), (16, 4, 64), seed=4)


def test_negative_scale(torch_cuda):
    _decode(torch_cuda, [100, 33], None, (8, 2, 128), seed=5, scale=-0.2)


def test_bad_tables_are_skipped_and_flagged(torch_cuda):
    torch = torch_cuda
    from paper_2603_03310_amd import ent
    from paper_2603_03310_amd.runner import Decoder
    rng = np.random.default_rng(6)
    H, d, P = 2, 64, 6
    kc, ks, vc, vs = _cache(torch, rng, P, H, d, True)
    q, _ = to_dev(torch, rng.normal(size=(2, H, d)))
    good, bad = torch.zeros(2, H, d, device="cuda:0"), torch.zeros(2, H, d, device="cuda:0")
    lens = _i32(torch, [80, 16])
    kept = np.full((2, 64), -1)
    kept[0, :5] = np.arange(5)
    kept[1, 0] = 0
    with Decoder(**config(H, H, d, num_pool_blocks=P)) as dec:
        for out, row, ids in ((good, [3, 1, 0, 2, 4], [0, 2, 4]), (bad, [3, 99, 0, -5, 4], range(5))):
            tab = np.full((2, 64), -1)
            tab[0, :5] = row
            tab[1, 0] = 5
            k = kept.copy()
            k[0, :len(ids)] = list(ids)
            ent.ent_sparse_paged_decode_q8(dec.ctx, 2, q, kc, vc, ks, vs, _i32(torch, tab), lens,
                                           _i32(torch, k), _i32(torch, [len(ids), 1]), out)
            torch.cuda.synchronize()
            assert dec.device_status() == (ent.ENT_DEV_BAD_TABLE if out is bad else 0)
    # The same three blocks; in other groups, so equal but for the order of a few sums.
    assert torch.allclose(good, bad, rtol=1e-5, atol=1e-6)


@pytest.mark.parametrize("heads", [(2, 128), (3, 64), (16, 128)], ids=str)
def test_append_equals_oracle_and_store(torch_cuda, heads):
    """40 appends to sequences of different lengths, values that outgrow their block's range:
    caches, scales, means and lengths as the oracle's and, token by token, the store's."""
    torch = torch_cuda
    from paper_2603_03310_amd.runner import Decoder
    H, d = heads
    rng = np.random.default_rng(d + H)
    B, maxb = 5, 6
    lens = np.array([0, 1, 15, 16, 37])
    P = B * maxb
    tab = rng.permutation(P).reshape(B, maxb)
    kc, ks, vc, vs = _cache(torch, rng, P, H, d, True)
    mine = [kc, vc, ks, vs, torch.zeros(P, H, d, device="cuda:0")]
    other = [t.clone() for t in mine]
    table = OP.e4m3_values()
    kv, vv = table[kc.cpu().numpy()], table[vc.cpu().numpy()]
    wk, wv, wm = ks.cpu().numpy(), vs.cpu().numpy(), np.zeros((P, H, d))
    dl, dt = _i32(torch, lens), _i32(torch, tab)
    with Decoder(**config(H, H, d, max_blocks_per_seq=maxb, num_pool_blocks=P)) as dec:
        for step in range(40):
            x = rng.normal(size=(2, B, H, d)) * np.exp2(rng.integers(-4, 5, (2, B, H, 1)))
            rows, val = to_dev(torch, x)
            slots = np.array([tab[b, n // 16] * 16 + n % 16 for b, n in enumerate(lens)])
            dec.append(B, rows[0], rows[1], dt, dl, mine[0], mine[1], mine[4], k_scale=mine[2],
                       v_scale=mine[3])
            dec.store(rows[0], rows[1], torch.tensor(slots, device="cuda:0"), other[0], other[1],
                      other[4], other[2], other[3])
            OP.store8(kv, vv, wk, wv, wm, slots, val[0], val[1])
            lens = lens + 1
        torch.cuda.synchronize()
        assert dec.device_status() == 0
    for a, b in zip(mine, other):
        assert torch.equal(a, b)
    assert np.array_equal(table[kc.cpu().numpy()], kv) and np.array_equal(table[vc.cpu().numpy()], vv)
    assert np.array_equal(ks.cpu().numpy(), wk) and np.array_equal(vs.cpu().numpy(), wv)
    assert np.allclose(mine[4].cpu().numpy(), wm, rtol=2.0 ** -22, atol=0)
    assert np.array_equal(dl.cpu().numpy(), lens)


def test_append_without_room(torch_cuda):
    torch = torch_cuda
    from paper_2603_03310_amd import ent
    from paper_2603_03310_amd.runner import Decoder
    rng = np.random.default_rng(11)
    kc, ks, vc, vs = _cache(torch, rng, 4, 2, 64, True)
    before = [t.clone() for t in (kc, vc, ks, vs)]
    x = torch.ones(3, 2, 64, dtype=torch.bfloat16, device="cuda:0")
    ksum = torch.zeros(4, 2, 64, device="cuda:0")
    for n, row, flag in ((32, [0, 1], ent.ENT_DEV_CACHE_FULL), (-1, [0, 1], ent.ENT_DEV_BAD_CTXLEN),
                         (3, [4, 1], ent.ENT_DEV_BAD_TABLE), (3, [-1, 1], ent.ENT_DEV_BAD_TABLE)):
        lens = _i32(torch, [n] * 3)
        with Decoder(**config(2, 2, 64, max_blocks_per_seq=2, num_pool_blocks=4)) as dec:
            dec.append(3, x, x, _i32(torch, [row] * 3), lens, kc, vc, ksum, k_scale=ks, v_scale=vs)
            assert dec.device_status() == flag
        assert (lens == n).all() and all(torch.equal(a, b) for a, b in zip(before, (kc, vc, ks, vs)))
