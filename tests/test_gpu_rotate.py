"""ent_qk_norm_rope against the float64 oracle: head shapes, types, strides, pairs,
partial rotation, positions of prompts and of steps, rows that are left alone,
in place, values that are not finite, and refusals."""
import numpy as np
import pytest

from oracle import rotate as OR
from tests.prompt_data import BF16_HALF, U32, config, host, to_dev
from tests.test_gpu_parity import torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu


def bound(out, size, dtype):
    """r: 1/2 of the sum of squares' (d <= 128: at most 8 additions in a lane, 5 across, a
    product: 14 roundings), mean and eps 1, root 2; gain times cosine 1, cosine and sine 2
    and their angle's pi / 2 (rounded within one turn); product, sum and product by r 3: 17
    roundings of |y_a| + |y_b| at the most, and the output's own."""
    return 17 * U32 * size + (BF16_HALF if dtype == "bf16" else U32) * np.abs(out) + 1e-37


def freqs(rot):
    return (500000.0 ** (-np.arange(rot // 2) * 2 / max(rot, 1))).astype(np.float32)


def run(torch, c, q, k, prm, starts, ctx, in_place=False, T=None, **kw):
    from paper_2603_03310_amd.runner import Decoder
    i32 = lambda x: None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda:0")  # noqa: E731
    outs = (q, k) if in_place else tuple(torch.full(x.shape, -7.0, dtype=x.dtype, device="cuda:0") for x in (q, k))
    B = len(starts) - 1 if starts is not None else q.shape[0]
    with Decoder(**c) as dec:
        dec.rotate(B, prm, q, k, *outs, starts=i32(starts), ctx_lens=i32(ctx), **kw)
        torch.cuda.synchronize()
        return host(outs[0]), host(outs[1]), dec.device_status()


def check(got, x, old, pos, gain, f, eps, rot, adjacent, dtype):
    ref, size = OR.norm_rope(x, pos, gain, f, eps, rot, adjacent)
    left = pos < 0
    assert np.array_equal(got[left], old[left])
    err = np.abs(got - ref)[~left]
    assert (err <= bound(ref, size, dtype)[~left]).all(), float((err / bound(ref, size, dtype)[~left]).max())


CASES = [  # Hq, Hkv, d, dtype, rot, adjacent, norms of (q, k)
    (32, 8, 128, "bf16", 128, False, (1, 1)), (32, 8, 128, "bf16", 128, True, (1, 1)),
    (64, 8, 128, "bf16", 64, False, (0, 1)), (10, 10, 128, "bf16", 48, False, (1, 0)),
    (6, 6, 64, "bf16", 64, False, (1, 1)), (16, 1, 64, "bf16", 16, False, (0, 0)),
    (16, 4, 64, "bf16", 48, True, (1, 1)), (8, 2, 64, "f32", 64, False, (1, 1)),
    (8, 2, 64, "f32", 32, True, (1, 1)), (5, 5, 128, "f32", 128, False, (1, 1)),
    (4, 1, 128, "f32", 80, False, (0, 0)), (4, 2, 64, "f32", 0, False, (1, 1)),
    (1, 1, 64, "bf16", 0, False, (0, 1)), (1, 1, 128, "f32", 112, False, (1, 1))]


def data(torch, rng, T, Hq, Hkv, d, dtype, fused):
    if fused:
        rows, x = to_dev(torch, rng.normal(size=(T, Hq + 2 * Hkv, d)) * np.exp(rng.normal(size=(T, 1, 1))), dtype)
        return rows[:, :Hq], rows[:, Hq:Hq + Hkv], x[:, :Hq], x[:, Hq:Hq + Hkv]
    q, qx = to_dev(torch, rng.normal(size=(T, Hq, d)), dtype)
    k, kx = to_dev(torch, rng.normal(size=(T, Hkv, d)) * 5, dtype)
    return q, k, qx, kx


def params(torch, rng, d, rot, adjacent, norms, eps=1e-5):
    from paper_2603_03310_amd import ent
    g = [rng.normal(size=d).astype(np.float32) + 1 if n else None for n in norms]
    dev = [None if x is None else torch.tensor(x, device="cuda:0") for x in g + [freqs(rot)]]
    return ent.make_qk_params(*dev, eps, rot, adjacent), g


@pytest.mark.parametrize("fused", [False, True], ids=["apart", "fused"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_prompts(torch_cuda, case, fused):
    torch = torch_cuda
    Hq, Hkv, d, dtype, rot, adjacent, norms = case
    rng = np.random.default_rng(sum(map(ord, str(case))))
    lens, ctx = [3, 0, 1, 40, 17, 0, 2], [0, 9, 131000, 5, 0, 0, 16384 * 8]
    starts = np.cumsum([0] + lens)
    T = int(starts[-1]) + 5
    q, k, qx, kx = data(torch, rng, T, Hq, Hkv, d, dtype, fused)
    prm, g = params(torch, rng, d, rot, adjacent, norms)
    c = config(Hq, Hkv, d, dtype, max_blocks_per_seq=8200)
    gq, gk, flags = run(torch, c, q, k, prm, starts, ctx)
    pos, _ = OR.positions(T, starts, ctx, 8200 * 16)
    assert flags == 0 and (pos[-5:] == -1).all()
    for got, x, gain in ((gq, qx, g[0]), (gk, kx, g[1])):
        check(got, x, np.full_like(got, -7.0), pos, gain, freqs(rot), 1e-5, rot, adjacent, dtype)


@pytest.mark.parametrize("case", [CASES[0], CASES[3], CASES[8], CASES[9]], ids=str)
@pytest.mark.parametrize("T", [1, 2, 63, 130])
def test_steps_and_in_place(torch_cuda, case, T):
    """One row per sequence, in place in one projection's rows: the values stay as they are."""
    torch = torch_cuda
    Hq, Hkv, d, dtype, rot, adjacent, norms = case
    rng = np.random.default_rng(T)
    q, k, qx, kx = data(torch, rng, T, Hq, Hkv, d, dtype, True)
    whole = q._base if q._base is not None else q
    before = host(whole)
    ctx = rng.integers(0, 1024, T)
    ctx[0] = 1024 if T > 1 else 7
    prm, g = params(torch, rng, d, rot, adjacent, norms)
    gq, gk, flags = run(torch, config(Hq, Hkv, d, dtype, max_batch=T), q, k, prm, None, ctx, in_place=True)
    assert flags == 0
    for got, x, gain in ((gq, qx, g[0]), (gk, kx, g[1])):
        check(got, x, x, ctx, gain, freqs(rot), 1e-5, rot, adjacent, dtype)
    assert np.array_equal(host(whole)[:, Hq + Hkv:], before[:, Hq + Hkv:])


def test_many_rows_and_requests(torch_cuda):
    """More requests than a wave has lanes, some of them empty; no lengths before."""
    torch = torch_cuda
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 9, 700) * (rng.random(700) < 0.6)
    starts = np.cumsum(np.concatenate([[0], lens]))
    T = int(starts[-1])
    q, k, qx, kx = data(torch, rng, T, 4, 2, 64, "bf16", False)
    prm, g = params(torch, rng, 64, 64, False, (1, 1))
    gq, gk, flags = run(torch, config(4, 2, 64, max_batch=700), q, k, prm, starts, None)
    pos, _ = OR.positions(T, starts, None, 1024)
    assert flags == 0 and pos.min() == 0
    check(gq, qx, qx, pos, g[0], freqs(64), 1e-5, 64, False, "bf16")
    check(gk, kx, kx, pos, g[1], freqs(64), 1e-5, 64, False, "bf16")


def test_bad_lengths_and_starts(torch_cuda):
    torch = torch_cuda
    from paper_2603_03310_amd import ent
    rng = np.random.default_rng(4)
    q, k, qx, kx = data(torch, rng, 12, 4, 4, 64, "f32", False)
    prm, g = params(torch, rng, 64, 64, False, (1, 1))
    starts, ctx = [0, 4, 8, 12], [0, 1025, 3]
    gq, _, flags = run(torch, config(4, 4, 64, "f32"), q, k, prm, starts, ctx)
    pos, bad = OR.positions(12, starts, ctx, 1024)
    assert bad and flags == ent.ENT_DEV_BAD_CTXLEN
    check(gq, qx, np.full_like(gq, -7.0), pos, g[0], freqs(64), 1e-5, 64, False, "f32")
    # Starts that no plan gives: every row is turned as some request's, or left alone.
    for bad_starts in ([5, 1, 1 << 30, -8], [-(1 << 31), (1 << 31) - 1, 0, 3], [99, 99, 99, 99]):
        gq, gk, _ = run(torch, config(4, 4, 64, "f32"), q, k, prm, bad_starts, [0, 0, 0])
        assert np.isfinite(gq).all() and np.isfinite(gk).all()


def test_values_not_finite_stay_in_their_head(torch_cuda):
    torch = torch_cuda
    rng = np.random.default_rng(5)
    for dtype in ("bf16", "f32"):
        q, k, _, _ = data(torch, rng, 3, 4, 2, 128, dtype, False)
        for norms in ((1, 1), (0, 0)):
            prm, _ = params(torch, rng, 128, 64, False, norms)
            c = config(4, 2, 128, dtype)
            good, _, _ = run(torch, c, q, k, prm, None, [3, 4, 5])
            q2 = q.clone()
            q2[1, 2, 40] = float("nan")
            q2[2, 0, 100] = float("inf")      # a dim that does not turn
            got, _, _ = run(torch, c, q2, k, prm, None, [3, 4, 5])
            same = np.ones((3, 4, 128), bool)
            if norms[0]:
                same[1, 2] = same[2, 0] = False
                assert np.isnan(got[1, 2]).all() and np.isnan(got[2, 0, 100])
            else:
                same[1, 2, [8, 40]] = same[2, 0, 100] = False
                assert np.isnan(got[1, 2, [8, 40]]).all() and got[2, 0, 100] == np.inf
            assert np.array_equal(got[same], good[same])


def test_another_stream_and_empty_calls(torch_cuda):
    torch = torch_cuda
    from paper_2603_03310_amd.runner import Decoder
    rng = np.random.default_rng(6)
    q, k, qx, _ = data(torch, rng, 5, 4, 2, 64, "bf16", False)
    prm, g = params(torch, rng, 64, 64, False, (1, 1))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    gq, _, _ = run(torch, config(4, 2, 64), q, k, prm, None, [1, 2, 3, 4, 5], stream=s)
    check(gq, qx, qx, np.arange(1, 6), g[0], freqs(64), 1e-5, 64, False, "bf16")
    with Decoder(**config(4, 2, 64)) as dec:
        out = torch.full_like(q, 3.0)
        dec.rotate(0, prm, q[:0], k[:0], out[:0], k[:0])
        dec.rotate(0, prm, q, k, out, torch.empty_like(k), starts=torch.zeros(1, dtype=torch.int32, device="cuda:0"))
        torch.cuda.synchronize()
        assert (out == 3.0).all().item()


def test_refusals(torch_cuda):
    torch = torch_cuda
    from paper_2603_03310_amd import ent
    from paper_2603_03310_amd.runner import Decoder
    rng = np.random.default_rng(7)
    rows, _ = to_dev(torch, rng.normal(size=(8, 12, 64)))
    q, k = rows[:, :4], rows[:, 4:6]
    qo, ko = torch.full((8, 4, 64), -7.0, dtype=q.dtype, device="cuda:0"), torch.empty((8, 2, 64), dtype=q.dtype, device="cuda:0")
    ctx = torch.zeros(8, dtype=torch.int32, device="cuda:0")
    prm, _ = params(torch, rng, 64, 64, False, (1, 1))
    f, g = prm.tensors[2], prm.tensors[0]

    def call(dec, p=prm, q=q, k=k, qo=qo, ko=ko, B=8, T=8, ldq=None, starts=None):
        ent.ent_qk_norm_rope(dec.ctx, B, T, p, q, ldq or 12 * 64, k, 12 * 64, starts, ctx, qo,
                             qo.stride(0), ko, ko.stride(0))

    mk = ent.make_qk_params
    inval, unsup = ent.ENT_E_INVAL, ent.ENT_E_UNSUPPORTED
    with Decoder(**config(4, 2, 64, max_batch=8)) as dec:
        for code, kw in [
                (inval, dict(p=mk(g, g, f, float("nan"), 64))), (inval, dict(p=mk(g, g, f, -1.0, 64))),
                (inval, dict(p=mk(g, g, f, 0.0, 80))), (inval, dict(p=mk(g, g, f, 0.0, -16))),
                (unsup, dict(p=mk(g, g, f, 0.0, 24))), (inval, dict(p=mk(g, g, None, 0.0, 64))),
                (inval, dict(T=7)), (inval, dict(B=9, T=9)), (inval, dict(ldq=4 * 64 - 8)),
                (inval, dict(ldq=4 * 64 + 4)), (inval, dict(T=-1, starts=ctx)),
                (unsup, dict(T=ent.ENT_MAX_PACKED_TOKENS + 1, starts=ctx)),
                (inval, dict(qo=rows[:, 1:5])), (inval, dict(ko=rows[:, 3:5])), (inval, dict(qo=rows[:, 4:8])),
                (inval, dict(qo=rows[:, 6:10], ko=rows[:, 9:11])), (inval, dict(q=q.data_ptr() + 2))]:
            with pytest.raises(ent.EntError) as e:
                call(dec, **kw)
            assert e.value.code == code, (kw, str(e.value))
        with pytest.raises(ent.EntError):
            dec.rotate(8, prm, q, k, qo[:, :, ::2], ko, ctx_lens=ctx)
        torch.cuda.synchronize()
        assert (qo == -7.0).all().item()
        # Beside each other in one projection's rows is no overlap.
        call(dec, qo=rows[:, 6:10], ko=rows[:, 10:12])
        torch.cuda.synchronize()


def test_offsets_past_32_bits(torch_cuda):
    """Rows that lie more than 2^32 elements into their buffers, at the largest row stride."""
    torch = torch_cuda
    rng = np.random.default_rng(13)
    T, ld = 300, 1 << 24
    buf = torch.empty((T - 1) * ld + 8 * 64, dtype=torch.bfloat16, device="cuda:0")
    rows = torch.as_strided(buf, (T, 8, 64), (ld, 64, 1))
    q, k, qx, kx = data(torch, rng, T, 2, 2, 64, "bf16", False)
    rows[:, :2], rows[:, 2:4] = q, k
    prm, g = params(torch, rng, 64, 64, False, (1, 1))
    from paper_2603_03310_amd.runner import Decoder
    with Decoder(**config(2, 2, 64, max_batch=T)) as dec:
        ctx = torch.arange(T, dtype=torch.int32, device="cuda:0")
        dec.rotate(T, prm, rows[:, :2], rows[:, 2:4], rows[:, 4:6], rows[:, 6:8], ctx_lens=ctx)
        torch.cuda.synchronize()
    got = host(rows)
    check(got[:, 4:6], qx, got[:, 4:6], np.arange(T), g[0], freqs(64), 1e-5, 64, False, "bf16")
    check(got[:, 6:8], kx, got[:, 6:8], np.arange(T), g[1], freqs(64), 1e-5, 64, False, "bf16")
    assert np.array_equal(got[:, :2], qx) and np.array_equal(got[:, 2:4], kx)
