"""ent_token_logprobs against the float64 oracle: vocabularies, types, alignments, rows
split over workgroups and not, ties, masks, rows without a distribution, rows whose
largest logits lie side by side or far apart, skipped rows, and refusals."""
import numpy as np
import pytest

from oracle import logprobs as OL
from tests.prompt_data import U32, config
from tests.test_gpu_parity import torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu


def bounds(lp, h, V):
    """c = log2(e) / T off by 2 roundings and each t = c (z - M) by 2 more, relative to |t|; sums of
    V / 256 terms in a thread (at least; each exponential 2 roundings), their rescaling and the
    sums over threads 80 at the most; logarithm and products 4.  A token's |t| is at most
    |ln p| + ln V; the mean of |t| is at most H."""
    n, top = V / 256 + 80, np.log(V)
    return U32 * (n + 8 * (np.abs(lp) + top)), U32 * ((n + 20) * (1 + h) + 8 * top)


def run(torch, z, tokens, n_top, temp=None, t_cal=1.0, **kw):
    from paper_2603_03310_amd.runner import Decoder
    T, V = z.shape
    f = lambda *s: torch.full(s, -7.0, device="cuda:0")  # noqa: E731
    lp, h, top = f(T), f(T), f(T, n_top)
    ids = torch.full((T, n_top), -7, dtype=torch.int32, device="cuda:0")
    tk = None if tokens is None else torch.tensor(np.asarray(tokens), dtype=torch.int32, device="cuda:0")
    tp = None if temp is None else torch.tensor(np.asarray(temp), dtype=torch.float32, device="cuda:0")
    with Decoder(**config(8, 8, 64, vocab=V, log_v=20.0, t_cal=t_cal)) as dec:
        dec.logprobs(z, tk, None if tokens is None else lp, h, ids if n_top else None, top if n_top else None,
                     tp, **kw)
        torch.cuda.synchronize()
        flags = dec.device_status()
    return lp.cpu().numpy(), h.cpu().numpy(), ids.cpu().numpy(), top.cpu().numpy(), flags


def check(z, got, tokens, n_top, temp=None, t_cal=1.0):
    lp, h, ids, top, flags = got
    zh = z.double().cpu().numpy()
    V = zh.shape[1]
    want_flags = 0
    for t in range(len(zh)):
        tok = int(tokens[t]) if tokens is not None else 0
        if tok < 0:
            assert lp[t] == h[t] == -7.0 and (ids[t] == -7).all() and (top[t] == -7.0).all()
            continue
        want_flags |= 8 if tok >= V else 0
        # The product of two float32, as the definition has it.
        T = float(np.float32(1.0 if temp is None else temp[t])) * float(np.float32(t_cal))
        r = OL.token_logprobs(zh[t], tok, T, n_top)
        assert np.array_equal(ids[t], r[2]), (t, ids[t], r[2])
        if np.isnan(r[1]):
            assert np.isnan(h[t]) and np.isnan(top[t]).all() and (tokens is None or np.isnan(lp[t]))
            continue
        b = bounds(np.where(np.isinf(r[3]), 0, r[3]), r[1], V)
        assert abs(h[t] - r[1]) <= b[1], (t, h[t], r[1])
        fin = np.isfinite(r[3])
        assert np.array_equal(top[t][~fin], r[3][~fin].astype(np.float32))
        assert (np.abs(top[t][fin] - r[3][fin]) <= b[0][fin]).all()
        if tokens is not None:
            if tok >= V:
                assert np.isnan(lp[t])
            elif np.isinf(r[0]):
                assert lp[t] == r[0]
            else:
                assert abs(lp[t] - r[0]) <= bounds(r[0], r[1], V)[0], (t, lp[t], r[0])
    assert flags == want_flags


def rows(torch, rng, T, V, dtype, pad=0, first=0, scale=3.0):
    """Rows of V logits in a buffer whose rows are V + pad apart, from element `first` on."""
    x = rng.normal(size=(T, V + pad)) * scale
    for t in range(T):
        x[t, rng.integers(0, V, 4)] += rng.random(4) * 8
    buf = torch.zeros(first + T * (V + pad), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda:0")
    buf[first:] = torch.tensor(x.reshape(-1), device="cuda:0").to(buf.dtype)
    return buf[first:].view(T, V + pad)[:, :V]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 5, 33, 1000, 1024, 2049, 32000, 128256, 262144])
def test_vocabularies(torch_cuda, V, dtype):
    torch = torch_cuda
    rng = np.random.default_rng(V)
    n = min(V, [0, 1, 5, 20, 32][V % 5])
    for T in (1, 5):
        z = rows(torch, rng, T, V, dtype)
        tokens = rng.integers(0, V, T)
        tokens[0] = int(z[0].float().argmax())
        check(z, run(torch, z, tokens, n), tokens, n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 70, 1100])
@pytest.mark.parametrize("pad,first", [(0, 0), (1, 0), (3, 5), (8, 1)])
def test_alignments_temperatures_and_skipped_rows(torch_cuda, T, dtype, pad, first):
    torch = torch_cuda
    rng = np.random.default_rng(T + pad)
    V = 5003
    z = rows(torch, rng, T, V, dtype, pad, first)
    temp = rng.uniform(0.3, 3.0, T)
    tokens = rng.integers(0, V, T)
    if T > 1:
        tokens[::7] = -1
        tokens[3] = V
        tokens[4] = (1 << 31) - 1
    check(z, run(torch, z, tokens, 20, temp, 1.5), tokens, 20, temp, 1.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [3, 1030])
@pytest.mark.parametrize("V", [700, 70001])
def test_ties_masks_and_orders(torch_cuda, V, T, dtype):
    """Constant rows, few values, almost all masked, ascending, descending, and largest
    logits at the places of one thread (a workgroup's width apart)."""
    torch = torch_cuda
    rng = np.random.default_rng(V)
    if T > 3 and V > 70000:
        T = 1025
    z = rows(torch, rng, T, V, dtype)
    ninf = float("-inf")
    z[0] = 2.5
    z[1] = torch.tensor(rng.integers(0, 3, V), device="cuda:0")
    z[2] = ninf
    z[2, [V - 1, 17, 300]] = torch.tensor([1.0, 1.0, -3.0], device="cuda:0").to(z.dtype)
    if T > 3:
        z[3] = torch.arange(V, device="cuda:0") / 64
        z[4] = -torch.arange(V, device="cuda:0") / 64
        z[5, ::1024] = 50.0 + torch.arange(len(z[5, ::1024]), device="cuda:0").to(z.dtype)
        z[6, ::2048] = 50.0
        z[7] = ninf
        z[7, V // 2] = -1e30 if dtype == "f32" else -1e4
        z[8] = torch.where(torch.arange(V, device="cuda:0") % 2 == 0, 0.0, -0.0)
        z[9, :] = -3.0e38 if dtype == "f32" else -3.0e4
        z[10] = torch.arange(V, device="cuda:0") % 2048
        z[11, ::64] = 30.0
        z[12] = (torch.arange(V, device="cuda:0") % 1024 == 5) * 40.0 + torch.rand(V, device="cuda:0")
    tokens = np.full(T, 17)
    for n in (1, 32):
        got = run(torch, z, tokens, n)
        check(z, got, tokens, n)


@pytest.mark.parametrize("T,V", [(1, 1000000), (1025, 40000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_candidates_than_are_ranked_at_once(torch_cuda, T, V, dtype):
    """31 of a workgroup's 256 places hold logits that are all above the others' largest."""
    torch = torch_cuda
    rng = np.random.default_rng(1)
    z = rows(torch, rng, T, V, dtype)
    place = torch.arange(V, device="cuda:0") // (4 if dtype == "f32" else 8) % 256
    for t in range(0, T, 100):
        z[t] = torch.where(place < 31, 20.0, 0.0) + torch.rand(V, device="cuda:0")
    tokens = rng.integers(0, V, T)
    got = run(torch, z, tokens, 32)
    check(z[::25], [x[::25] for x in got[:4]] + [got[4]], tokens[::25], 32)


@pytest.mark.parametrize("T", [2, 1030])
def test_rows_without_a_distribution(torch_cuda, T):
    torch = torch_cuda
    rng = np.random.default_rng(2)
    for dtype in ("f32", "bf16"):
        for bad in (float("nan"), float("inf")):
            z = rows(torch, rng, T, 9001, dtype)
            z[0, 5000] = bad
            z[1] = float("-inf")
            if T > 2:
                z[2, 0] = z[2, 9000] = bad
                z[4] = bad
            tokens = np.arange(T)
            check(z, run(torch, z, tokens, 5), tokens, 5)


def test_without_tokens_and_outputs_left_out(torch_cuda):
    torch = torch_cuda
    from paper_2603_03310_amd import ent
    from paper_2603_03310_amd.runner import Decoder
    rng = np.random.default_rng(3)
    z = rows(torch, rng, 9, 3001, "f32")
    check(z, run(torch, z, None, 5), None, 5)
    lp = torch.full((9,), -7.0, device="cuda:0")
    with Decoder(**config(8, 8, 64, vocab=3001, log_v=20.0)) as dec:
        dec.logprobs(z, torch.zeros(9, dtype=torch.int32, device="cuda:0"), lp)
        torch.cuda.synchronize()
        want = [OL.token_logprobs(r, 0, 1.0, 0)[0] for r in z.double().cpu().numpy()]
        assert np.abs(lp.cpu().numpy() - want).max() < 1e-4
        ent.ent_token_logprobs(dec.ctx, 0, None, 0, 3001, None, None, None, None)


def test_same_bits_every_time(torch_cuda):
    torch = torch_cuda
    rng = np.random.default_rng(4)
    z = rows(torch, rng, 33, 50001, "bf16")
    tokens = rng.integers(0, 50001, 33)
    a = run(torch, z, tokens, 20)
    for _ in range(3):
        for x, y in zip(a[:4], run(torch, z, tokens, 20)[:4]):
            assert np.array_equal(x, y)


def test_refusals(torch_cuda):
    torch = torch_cuda
    from paper_2603_03310_amd import ent
    from paper_2603_03310_amd.runner import Decoder
    z = torch.zeros((4, 50), device="cuda:0")
    lp, tk = torch.full((4,), -7.0, device="cuda:0"), torch.zeros(4, dtype=torch.int32, device="cuda:0")
    ids, top = torch.zeros((4, 33), dtype=torch.int32, device="cuda:0"), torch.zeros((4, 33), device="cuda:0")
    inval, unsup = ent.ENT_E_INVAL, ent.ENT_E_UNSUPPORTED
    with Decoder(**config(8, 8, 64, vocab=50, log_v=20.0)) as dec:
        for code, kw in [(inval, dict(kind=2)), (inval, dict(n=-1)), (inval, dict(n=51)), (unsup, dict(n=33)),
                         (inval, dict(ld=49)), (inval, dict(T=-1)), (unsup, dict(T=ent.ENT_MAX_PACKED_TOKENS + 1)),
                         (inval, dict(z=None)), (inval, dict(tk=None)), (inval, dict(n=5, ids=None)),
                         (inval, dict(z=z.data_ptr() + 2))]:
            a = dict(dict(T=4, z=z, kind=0, ld=50, tk=tk, n=0, ids=ids), **kw)
            with pytest.raises(ent.EntError) as e:
                ent.ent_token_logprobs(dec.ctx, a["T"], a["z"], a["kind"], a["ld"], a["tk"], None, lp, None,
                                       a["n"], a["ids"], top)
            assert e.value.code == code, (kw, str(e.value))
        h = torch.full((4,), -7.0, device="cuda:0")
        for kw in (dict(entropy=lp), dict(temp=lp), dict(entropy=h, temp=h), dict(top_logprobs=lp), dict(top_ids=tk),
                   dict(entropy=z), dict(top_ids=ids, top_logprobs=ids)):
            a = dict(dict(entropy=None, temp=None, top_ids=ids, top_logprobs=top), **kw)
            with pytest.raises(ent.EntError) as e:
                ent.ent_token_logprobs(dec.ctx, 4, z, 0, 50, tk, a["temp"], lp, a["entropy"], 1, a["top_ids"],
                                       a["top_logprobs"])
            assert e.value.code == inval and "aliases" in str(e.value), kw
        with pytest.raises(ent.EntError):
            dec.logprobs(z.double(), tk, lp)
        with pytest.raises(ent.EntError):
            dec.logprobs(z.t().contiguous().t(), tk, lp)
        torch.cuda.synchronize()
        assert (lp == -7.0).all().item() and (h == -7.0).all().item()


def test_offsets_past_32_bits(torch_cuda):
    """Rows that lie more than 2^32 elements into their buffer."""
    torch = torch_cuda
    rng = np.random.default_rng(12)
    V, ld, T = 1001, 1 << 30, 6
    buf = torch.empty((T - 1) * ld + V, dtype=torch.bfloat16, device="cuda:0")
    z = torch.as_strided(buf, (T, V), (ld, 1))
    z.copy_(torch.tensor(rng.normal(size=(T, V)) * 3, device="cuda:0"))
    tokens = rng.integers(0, V, T)
    check(z, run(torch, z, tokens, 5), tokens, 5)


def test_two_graphs_and_another_stream(torch_cuda):
    """Two graphs of one context, with rows in parts and rows that are not, replayed in turn with
    eager calls between; and a call on another stream."""
    torch = torch_cuda
    from paper_2603_03310_amd.runner import Decoder
    rng = np.random.default_rng(14)
    V = 40001
    zs = [rows(torch, rng, 3, V, "f32"), rows(torch, rng, 1030, V, "bf16")]
    tk = [torch.tensor(rng.integers(0, V, len(z)), dtype=torch.int32, device="cuda:0") for z in zs]
    f = lambda *s: torch.zeros(*s, device="cuda:0")  # noqa: E731
    outs = [(f(len(z)), f(len(z)), torch.zeros((len(z), 7), dtype=torch.int32, device="cuda:0"), f(len(z), 7)) for z in zs]
    with Decoder(**config(8, 8, 64, vocab=V, log_v=20.0)) as dec:
        graphs, want = [], []
        for z, t, o in zip(zs, tk, outs):
            dec.logprobs(z, t, *o)
            torch.cuda.synchronize()
            want.append([x.clone() for x in o])
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=torch.cuda.Stream()):
                dec.logprobs(z, t, *o)
            graphs.append(g)
        for _ in range(3):
            for i in (0, 1, 1, 0):
                for x in outs[i]:
                    x.zero_()
                graphs[i].replay()
                torch.cuda.synchronize()
                assert all(torch.equal(x, w) for x, w in zip(outs[i], want[i]))
                dec.logprobs(zs[1 - i][:2], tk[1 - i][:2], *(x[:2] for x in outs[1 - i]))
                torch.cuda.synchronize()
        s = torch.cuda.Stream()
        for x in outs[0]:
            x.zero_()
        s.wait_stream(torch.cuda.current_stream())
        dec.logprobs(zs[0], tk[0], *outs[0], stream=s)
        s.synchronize()
        assert all(torch.equal(x, w) for x, w in zip(outs[0], want[0]))
