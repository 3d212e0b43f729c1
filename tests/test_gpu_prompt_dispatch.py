"""ent_prompt_attention in each of its forms (the splits of rows and keys over a workgroup's
waves, which the launch takes by the number of rows): scales of either sign and zero,
infinities and NaN that a row does not see, padding, empty requests, garbage in starts.
Each case first asserts that it lands in the form that it is meant for."""
import numpy as np
import pytest

from oracle import prompt as OP
from tests.prompt_data import attention_bound, config, host
from tests.test_gpu_parity import torch_cuda  # noqa: F401
from tests.test_gpu_prompt_attention import _check, _run

pytestmark = pytest.mark.gpu

MIXED = [5, 0, 410, 130, 0, 60]            # 605 tokens: more than 96 a request
SHORT = [33, 0, 31, 150, 17, 64, 1, 65, 7, 95]
PAD, LONG = 9, 2                           # padding rows; MIXED's long request
# form, heads (Hq, Hkv, d), lengths
BF16 = [("small", (16, 4, 128), SHORT), ("small", (16, 1, 64), SHORT),
        ("quarter", (16, 4, 128), MIXED), ("quarter", (16, 1, 64), MIXED), ("quarter", (8, 8, 128), MIXED),
        ("half", (32, 8, 128), MIXED), ("half", (32, 32, 64), MIXED), ("half", (32, 2, 64), MIXED),
        ("whole", (64, 8, 128), MIXED), ("whole", (64, 16, 64), MIXED), ("whole", (128, 8, 128), MIXED)]
F32 = [("quarter", (16, 4, 128), MIXED), ("quarter", (32, 8, 64), MIXED),
       ("half", (64, 8, 128), MIXED), ("half", (64, 32, 64), MIXED),
       ("whole", (128, 16, 128), MIXED), ("whole", (128, 32, 64), MIXED)]
CASES = [("bf16",) + c for c in BF16] + [("f32",) + c for c in F32]


def _form(torch, dtype, heads, lens, pad):
    """The launch's rule: which form a call of these sizes takes."""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    T, B = sum(lens) + pad, len(lens)
    rows = T * heads[0]
    if dtype == "f32":
        return "whole" if rows >= 256 * cus else "half" if rows >= 96 * cus else "quarter"
    if T <= 96 * B:
        return "small"
    if rows <= 64 * cus:
        return "quarter"
    return "half" if rows <= 128 * cus or (rows < 256 * cus and T >= 1024 * B) else "whole"


def _go(torch, dtype, form, heads, lens, **kw):
    assert _form(torch, dtype, heads, lens, PAD) == form
    print(f"[prompt] {dtype} {form} {heads} {lens} {sorted(kw)}", flush=True)
    return _run(torch, lens, heads, dtype, pad=PAD, **kw)


@pytest.mark.parametrize("scale", [-0.11, 0.0, 0.9, None])
@pytest.mark.parametrize("dtype,form,heads,lens", CASES, ids=str)
def test_scales(torch_cuda, dtype, form, heads, lens, scale):
    _check(*_go(torch_cuda, dtype, form, heads, lens, scale=scale, seed=11), dtype)


@pytest.mark.parametrize("what", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("dtype,form,heads,lens", CASES, ids=str)
def test_what_a_row_does_not_see(torch_cuda, dtype, form, heads, lens, what):
    """One token of a request has a value (and where `what` is a NaN, a key) that is not
    finite: first, inside, in the tile that a late stretch of rows sees in part, and last."""
    b = lens.index(max(lens))
    first, n = sum(lens[:b]), lens[b]
    for at in sorted({first, first + 77, first + n - n // 4, first + n - 1}):
        def spoil(q, k, v, starts):
            k[at, 0] = what if np.isnan(what) else k[at, 0]
            v[at, :, 3:9] = what
            q[starts[-1]:] = k[starts[-1]:] = v[starts[-1]:] = np.nan
        out, ls, starts, data, d = _go(torch_cuda, dtype, form, heads, lens, spoil=spoil, seed=at)
        q, k, v, sc = data
        E, end, G = int(starts[-1]), first + n, heads[0] // heads[1]
        o, l = host(out), host(ls)
        q, k, v = (np.where(np.isfinite(x), x, 0.0) for x in (q, k, v))
        ref, _, mass, span = OP.attention(q, k, v, starts, sc)
        bound = attention_bound(ref[:E], mass[:E], span[:E], d, n, dtype)
        near = np.abs(o[:E] - ref[:E]) <= bound
        hit = np.zeros(E, bool)
        hit[at:end] = True
        assert near[~hit].all() and np.isfinite(l[:E][~hit]).all()
        assert (o[E:] == -7).all() and (l[E:] == -7).all()
        if np.isnan(what):
            assert np.isnan(o[at:end, :, 3:9]).all()
            # The key of KV head 0 enters its query heads' sums, the others' not.
            assert np.isnan(o[at:end, :G]).all() and np.isnan(l[at:end, :G]).all()
            assert np.isfinite(l[at:end, G:]).all()
            assert near[at:end, G:, :3].all() and near[at:end, G:, 9:].all()
        else:
            assert (o[at:end, :, 3:9] == what).all() and np.isfinite(l[at:end]).all()
            assert near[at:end, :, :3].all() and near[at:end, :, 9:].all()


@pytest.mark.parametrize("dtype,form,heads,lens", CASES, ids=str)
def test_garbage_in_starts_and_repeats(torch_cuda, dtype, form, heads, lens):
    """Starts of any value keep inside the packed rows (the rows before and behind those of the
    call keep their sentinel); a good batch afterwards is right, and the same bits every time."""
    torch = torch_cuda
    from paper_2603_03310_amd.runner import Decoder
    Hq, Hkv, d = heads
    assert _form(torch, dtype, heads, lens, PAD) == form
    print(f"[prompt] {dtype} {form} {heads} garbage", flush=True)
    edt = torch.bfloat16 if dtype == "bf16" else torch.float32
    T, B = sum(lens) + PAD, len(lens)
    rng = np.random.default_rng(12)
    x = torch.randn(T + 2, Hq + 2 * Hkv, d, device="cuda:0").to(edt)
    buf = torch.full((T + 2, Hq, d), -7.0, dtype=edt, device="cuda:0")
    mid, out = x[1:-1], buf[1:-1]
    args = (mid[:, :Hq], mid[:, Hq:Hq + Hkv], mid[:, Hq + Hkv:])
    good = np.concatenate([[0], np.cumsum(lens)])
    bad = [rng.permutation(good), good[::-1].copy(), good + 10 ** 6, good - 10 ** 6,
           rng.integers(-2 ** 31, 2 ** 31, B + 1), np.where(np.arange(B + 1) % 2, T, 0)]
    with Decoder(**config(Hq, Hkv, d, dtype)) as dec:
        for st in bad:
            dec.prompt(B, *args, torch.tensor(st, dtype=torch.int32, device="cuda:0"), out)
        torch.cuda.synchronize()
        assert (buf[0] == -7).all() and (buf[-1] == -7).all()
        st = torch.tensor(good, dtype=torch.int32, device="cuda:0")
        runs = []
        for _ in range(5):
            out.fill_(-7.0)
            dec.prompt(B, *args, st, out)
            runs.append(out.clone())
        torch.cuda.synchronize()
        assert dec.device_status() == 0
    assert all(torch.equal(r, runs[0]) for r in runs)
    q, k, v = (host(t) for t in args)
    _check(runs[0], None, good, (q, k, v, float(np.float32(1.0 / d ** 0.5))), d, dtype)
