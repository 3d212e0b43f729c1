"""ent_prompt_attention against the float64 oracle: types, head groups, request
lengths from none to several tiles and across them, strides, padding, scales of
either sign and zero, large scores, and infinities and NaN in places that a row
does not see."""
import numpy as np
import pytest

from oracle import prompt as OP
from tests.prompt_data import attention_bound, config, host, lse_bound, to_dev
from tests.test_gpu_parity import torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

HEADS = [(8, 8, 64), (4, 2, 128), (8, 2, 128), (8, 1, 64), (16, 1, 128), (16, 2, 64), (12, 6, 64)]
LENGTHS = {
    "one": [1],
    "short": [1, 2, 0, 3, 15, 16, 17, 0, 1, 1],
    "empty_ends": [0, 5, 0],
    "tile": [64],
    "tile_less": [63, 65],
    "ragged": [130, 1, 0, 255, 33, 7, 200],
    "long": [700],
}


def _run(torch, lens, heads, dtype, pad=0, fused=True, scale=None, amp=1.0, seed=0, spoil=None,
         lse=True, **kw):
    """Runs one batch; returns what it gave and what it may give.  spoil(q, k, v, starts)
    changes the float64 inputs before they go to the GPU."""
    from paper_2603_03310_amd.runner import Decoder
    Hq, Hkv, d = heads
    rng = np.random.default_rng(seed)
    starts = np.concatenate([[0], np.cumsum(lens)])
    T = int(starts[-1]) + pad
    rows = rng.normal(size=(T, Hq + 2 * Hkv, d)) * amp
    if spoil:
        spoil(rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:], starts)
    dev, val = to_dev(torch, rows, dtype)
    q, k, v = dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:]
    if not fused:
        q, k, v = (t.contiguous() for t in (q, k, v))
    cfg = config(Hq, Hkv, d, dtype, **kw)
    if scale is not None:
        cfg["scale"] = scale
    out = torch.full((T, Hq, d), -7.0, dtype=dev.dtype, device="cuda:0")
    ls = torch.full((T, Hq), -7.0, device="cuda:0") if lse else None
    st = torch.tensor(starts, dtype=torch.int32, device="cuda:0")
    with Decoder(**cfg) as dec:
        dec.prompt(len(lens), q, k, v, st, out, ls)
        torch.cuda.synchronize()
        assert dec.device_status() == 0
    sc = float(np.float32(cfg["scale"]))
    return out, ls, starts, (val[:, :Hq], val[:, Hq:Hq + Hkv], val[:, Hq + Hkv:], sc), d


def _check(out, ls, starts, data, d, dtype):
    q, k, v, sc = data
    ref, rl, mass, span = OP.attention(q, k, v, starts, sc)
    E = int(starts[-1])
    n = int(np.diff(starts).max())
    o = host(out)
    assert (o[E:] == -7).all()
    bound = attention_bound(ref[:E], mass[:E], span[:E], d, n, dtype)
    bad = np.abs(o[:E] - ref[:E]) > bound
    assert not bad.any() and not np.isnan(o[:E]).any(), \
        f"{bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(o[:E] - ref[:E]) / bound)} of the bound"
    if ls is not None:
        l = host(ls)
        assert (l[E:] == -7).all()
        assert (np.abs(l[:E] - rl[:E]) <= lse_bound(rl[:E], span[:E], d, n)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", LENGTHS.values(), ids=LENGTHS.keys())
@pytest.mark.parametrize("heads", HEADS[:5], ids=str)
def test_lengths_and_groups(torch_cuda, heads, lens, dtype):
    r = _run(torch_cuda, lens, heads, dtype, pad=3)
    _check(*r, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_many_heads_and_rows(torch_cuda, heads, dtype):
    """Enough rows that the larger tiles run (512 rows per compute unit)."""
    Hq, Hkv, d = heads
    rep = 4 if Hkv * d <= 512 else 1
    lens = [400 * 16 // Hq + 37, 1, 900]
    r = _run(torch_cuda, lens, (Hq * rep, Hkv * rep, d), dtype, fused=False, seed=3)
    _check(*r, dtype)


def test_large_tiles_bf16(torch_cuda):
    for heads, lens in [((64, 8, 128), [1500, 3, 777]), ((32, 32, 64), [2500, 1900]),
                        ((128, 8, 128), [1300])]:
        r = _run(torch_cuda, lens, heads, "bf16", seed=4)
        _check(*r, "bf16")


def test_every_split(torch_cuda):
    """Row counts on either side of the rules that split the keys over waves, with lengths
    that end in every part of a tile; batches of one to thousands of requests."""
    rng = np.random.default_rng(8)
    for heads, lens in [((4, 4, 128), [1024]), ((4, 4, 128), [1300, 77]), ((32, 8, 128), [250, 262, 1]),
                        ((16, 4, 64), [2030]), ((16, 1, 64), [1100, 1070]),
                        ((32, 8, 128), rng.integers(0, 12, 300).tolist()),
                        ((8, 2, 64), rng.integers(0, 4, 3000).tolist()),
                        ((64, 8, 64), rng.integers(1, 90, 70).tolist())]:
        r = _run(torch_cuda, lens, heads, "bf16", seed=len(lens), max_batch=4096,
                 max_blocks_per_seq=1)
        _check(*r, "bf16")


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 8, 64), (16, 1, 128), (16, 1, 64), (4, 4, 128)], ids=str)
def test_short_requests(torch_cuda, heads):
    """Around the mean length of 96 tokens under which workgroups are small."""
    for lens in ([96], [97], [1, 191], [2, 191], [95, 97, 96, 0, 192], [0, 400, 1, 1, 0, 65, 64, 63],
                 [33, 32, 31, 15, 16, 17, 1, 700, 0, 2]):
        r = _run(torch_cuda, lens, heads, "bf16", seed=sum(lens), pad=sum(lens) % 2)
        _check(*r, "bf16")


def test_every_split_fp32(torch_cuda):
    """The same on either side of the fp32 rules: 24576 and 65536 rows at 256 compute units."""
    for heads, lens in [((8, 8, 64), [1500, 1570]), ((8, 8, 64), [1500, 1571, 2]), ((32, 8, 128), [767]),
                        ((32, 8, 128), [700, 69]), ((16, 1, 64), [2049, 2046]), ((16, 1, 128), [1, 2050, 2046]),
                        ((64, 32, 64), [1, 700, 333])]:
        r = _run(torch_cuda, lens, heads, "f32", seed=len(lens), max_blocks_per_seq=1)
        _check(*r, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [-0.11, 0.0, 0.9])
def test_scales(torch_cuda, scale, dtype):
    r = _run(torch_cuda, [70, 5, 200], (8, 2, 64), dtype, scale=scale)
    _check(*r, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(torch_cuda, dtype):
    """Scores in the hundreds: one key holds nearly all the weight, the maximum jumps late."""
    r = _run(torch_cuda, [190, 64], (4, 2, 128), dtype, amp=5.0, seed=5)
    _check(*r, dtype)


def test_rising_scores(torch_cuda):
    """Every later key scores higher, in steps under and over the rescaling threshold."""
    for step in (0.02, 0.3, 3.0):
        def spoil(q, k, v, starts):
            q[:] = 1.0
            k[:] = (np.arange(len(k)) * step / 8.0)[:, None, None]
        r = _run(torch_cuda, [300], (8, 2, 64), "bf16", spoil=spoil)
        _check(*r, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", [np.inf, -np.inf, np.nan])
def test_what_a_row_does_not_see_does_not_touch_it(torch_cuda, what, dtype):
    """One token's key and value are not finite: earlier tokens and other requests stay
    exact; the token's own request is not finite from there on; padding may be anything."""
    lens, at = [40, 100, 3, 30], 40 + 37

    def spoil(q, k, v, starts):
        k[at, 0] = what if np.isnan(what) else k[at, 0]
        v[at, :, 3:9] = what
        q[starts[-1]:] = k[starts[-1]:] = v[starts[-1]:] = np.nan
    for heads in [(4, 4, 64), (16, 4, 128)]:
        out, ls, starts, data, d = _run(torch_cuda, lens, heads, dtype, pad=9, spoil=spoil)
        q, k, v, sc = data
        o = host(out)
        E = int(starts[-1])
        hit = np.zeros(len(o), bool)
        hit[at:140] = True
        v2 = np.where(np.isfinite(v), v, 0.0)
        k2 = np.where(np.isfinite(k), k, 0.0)
        q2 = np.where(np.isfinite(q), q, 0.0)
        ref, _, mass, span = OP.attention(q2, k2, v2, starts, sc)
        bound = attention_bound(ref[:E], mass[:E], span[:E], d, 100, dtype)
        ok = ~hit[:E]
        assert (np.abs(o[:E] - ref[:E])[ok] <= bound[ok]).all()
        assert (o[E:] == -7).all()
        bad = o[at:140, :, 3:9]
        if np.isnan(what):
            assert np.isnan(bad).all()
        else:
            assert (bad == what).all()
            assert (np.abs(o[at:140] - ref[at:140])[:, :, 9:] <= bound[at:140, :, 9:]).all()


def test_values_not_finite_in_whole_tiles(torch_cuda):
    """An infinite value far before the rows (in tiles seen whole) reaches all later rows."""
    def spoil(q, k, v, starts):
        v[10, 0, 5] = np.inf
    out, _, _, _, _ = _run(torch_cuda, [900], (8, 2, 128), "bf16", spoil=spoil)
    o = host(out)
    assert np.isfinite(o[:10]).all() and np.isinf(o[10:, :4, 5]).all()
    assert np.isfinite(o[:, 4:]).all() and np.isfinite(np.delete(o, 5, 2)).all()


def test_starts_out_of_order_stay_in_bounds(torch_cuda):
    """Garbage in starts (refused by no check, as it lies on the device): no row range
    leaves the packed rows, and the rows of a good batch are good afterwards."""
    torch = torch_cuda
    from paper_2603_03310_amd.runner import Decoder
    x = torch.randn(50, 8, 64, device="cuda:0").to(torch.bfloat16)
    out = torch.zeros_like(x)
    with Decoder(**config(8, 8, 64)) as dec:
        for st in ([0, 90, 20, 45, 1000], [-5, 10, 3, -9, 50], [7, 7, 7, 7, -1]):
            dec.prompt(4, x, x, x, torch.tensor(st, dtype=torch.int32, device="cuda:0"), out)
        torch.cuda.synchronize()
    _check(*_run(torch, [50], (8, 8, 64), "bf16"), "bf16")


def test_refusals(torch_cuda):
    torch = torch_cuda
    from paper_2603_03310_amd import ent
    from paper_2603_03310_amd.runner import Decoder
    x = torch.zeros(8, 4, 64, dtype=torch.bfloat16, device="cuda:0")
    st = torch.tensor([0, 8], dtype=torch.int32, device="cuda:0")
    out = torch.full_like(x, -7.0)
    with Decoder(**config(4, 4, 64, max_batch=2)) as dec:
        good = dict(B=1, T=8, q=x, ldq=256, k=x, ldk=256, v=x, ldv=256, starts=st, out=out, ldo=256)
        for bad, code in [(dict(B=3), ent.ENT_E_INVAL), (dict(B=-1), ent.ENT_E_INVAL),
                          (dict(T=-1), ent.ENT_E_INVAL),
                          (dict(T=ent.ENT_MAX_PACKED_TOKENS + 1), ent.ENT_E_UNSUPPORTED),
                          (dict(q=None), ent.ENT_E_INVAL), (dict(k=None), ent.ENT_E_INVAL),
                          (dict(v=None), ent.ENT_E_INVAL), (dict(starts=None), ent.ENT_E_INVAL),
                          (dict(out=None), ent.ENT_E_INVAL), (dict(ldq=248), ent.ENT_E_INVAL),
                          (dict(ldk=260), ent.ENT_E_INVAL), (dict(ldv=0), ent.ENT_E_INVAL),
                          (dict(ldo=255), ent.ENT_E_INVAL),
                          (dict(ldk=ent.ENT_MAX_ROW_STRIDE + 8), ent.ENT_E_INVAL),
                          (dict(q=x.data_ptr() + 2), ent.ENT_E_INVAL),
                          (dict(out=out.data_ptr() + 8), ent.ENT_E_INVAL),
                          (dict(out=x), ent.ENT_E_INVAL)]:
            with pytest.raises(ent.EntError) as e:
                ent.ent_prompt_attention(dec.ctx, **{**good, **bad})
            assert e.value.code == code, bad
        for nothing in (dict(B=0), dict(T=0)):
            ent.ent_prompt_attention(dec.ctx, **{**good, **nothing})
        torch.cuda.synchronize()
        assert (out == -7).all()


def test_another_stream_and_no_lse(torch_cuda):
    torch = torch_cuda
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        r = _run(torch, [300, 20], (8, 2, 128), "bf16", lse=False)
    _check(*r, "bf16")


def test_largest_batch(torch_cuda):
    """4096 requests of none to three tokens, in every split of either type."""
    lens = np.random.default_rng(9).integers(0, 4, 4096).tolist()
    for heads, dtype in [((2, 2, 128), "bf16"), ((4, 2, 128), "bf16"), ((16, 2, 128), "bf16"),
                         ((2, 2, 128), "f32"), ((6, 6, 64), "f32"), ((16, 1, 128), "f32")]:
        r = _run(torch_cuda, lens, heads, dtype, seed=9, max_batch=4096, max_blocks_per_seq=1)
        _check(*r, dtype)


def test_two_streams_at_once(torch_cuda):
    """One handle, two calls in flight: the operator keeps nothing in the handle."""
    torch = torch_cuda
    from paper_2603_03310_amd.runner import Decoder
    lens = [[1700, 3], [40, 900, 1]]
    xs = [torch.randn(sum(n), 16, 128, device="cuda:0").to(torch.bfloat16) for n in lens]
    st = [torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32, device="cuda:0") for n in lens]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    with Decoder(**config(8, 4, 128)) as dec:
        def go(i, out, stream):
            x = xs[i]
            dec.prompt(len(lens[i]), x[:, :8], x[:, 8:12], x[:, 12:], st[i], out, stream=stream)
        want = [torch.zeros(len(x), 8, 128, dtype=x.dtype, device="cuda:0") for x in xs]
        got = [[torch.zeros_like(w) for w in want] for _ in range(4)]
        for i in (0, 1):
            go(i, want[i], None)
        torch.cuda.synchronize()
        for pair in got:
            for i in (0, 1):
                go(i, pair[i], streams[i].cuda_stream)
        torch.cuda.synchronize()
        for pair in got:
            assert all(torch.equal(a, b) for a, b in zip(pair, want))


def test_the_wrapper_refuses_rows_in_pieces(torch_cuda):
    torch = torch_cuda
    from paper_2603_03310_amd import ent
    from paper_2603_03310_amd.runner import Decoder
    x = torch.zeros(8, 4, 64, dtype=torch.bfloat16, device="cuda:0")
    st = torch.tensor([0, 8], dtype=torch.int32, device="cuda:0")
    heads_first = torch.zeros(4, 8, 64, dtype=torch.bfloat16, device="cuda:0").transpose(0, 1)
    with Decoder(**config(4, 4, 64, num_pool_blocks=4)) as dec:
        good = dict(q=x, k=x.clone(), v=x.clone(), out=torch.zeros_like(x))
        kc, ksum = torch.zeros(4, 4, 16, 64, dtype=x.dtype, device="cuda:0"), torch.zeros(4, 4, 64, device="cuda:0")
        for name in good:
            for bad in (heads_first, x[:7].clone(), x[:, :2].clone(), torch.zeros_like(x).mT):
                with pytest.raises(ent.EntError) as e:
                    dec.prompt(1, **{**good, name: bad}, starts=st)
                assert e.value.code == ent.ENT_E_INVAL
        slots = torch.arange(8, device="cuda:0")
        for kw in (dict(k=heads_first), dict(v=x[:7]), dict(slots=slots[:7])):
            with pytest.raises(ent.EntError):
                dec.store(**{**dict(k=x, v=x, slots=slots, k_cache=kc, v_cache=kc, ksum=ksum), **kw})
        dec.prompt(1, **good, starts=st)
        torch.cuda.synchronize()
