"""ent_qk_norm_rope where a wave takes all steps of a row (more than 4096 rows) and more of
them than are in flight together, with the queries' gains and then the keys': every element
type, head size and pairing, below and above the size from which on rows take no places in the
caches (some 150 MB read and written), in place and apart.  Every row against the formula in 64 bits."""
import numpy as np
import pytest

from oracle import rotate as OR
from tests.prompt_data import BF16_HALF, U32, config
from tests.test_gpu_parity import torch_cuda  # noqa: F401
from tests.test_gpu_rotate import freqs, params

pytestmark = pytest.mark.gpu

# Nine steps a row and more, six at the most in flight; the last one of queries and of keys
# with lanes past the last head.
HEADS = {("bf16", 128): (22, 11), ("bf16", 64): (44, 22), ("f32", 128): (11, 11), ("f32", 64): (22, 11)}
PAIRS = {"halves": lambda d: (d, False), "any": lambda d: (d // 2, False), "adjacent": lambda d: (d, True),
         "adjacent_some": lambda d: (48, True)}


def formula(torch, x, pos, gain, f, eps, rot, adjacent):
    """What oracle.rotate.norm_rope returns, for many rows."""
    y = x.double()
    if gain is not None:
        y = y * torch.tensor(gain, device=x.device).double() / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
    w = pos.double()[:, None] * torch.tensor(f, device=x.device).double()
    c, s = torch.cos(w)[:, None], torch.sin(w)[:, None]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if adjacent else (slice(0, rot // 2), slice(rot // 2, rot))
    out, size = y.clone(), y.abs()
    out[..., a] = y[..., a] * c - y[..., b] * s
    out[..., b] = y[..., b] * c + y[..., a] * s
    size[..., a] = size[..., b] = y[..., a].abs() + y[..., b].abs()
    return out, size


@pytest.mark.parametrize("T,norms", [(4201, (1, 1)), (10001, (1, 1)), (4199, (1, 0)), (9999, (0, 1))], ids=str)
@pytest.mark.parametrize("pairs", list(PAIRS))
@pytest.mark.parametrize("dtype,d", list(HEADS), ids=str)
def test_rows_of_many_steps(torch_cuda, dtype, d, pairs, T, norms):
    torch = torch_cuda
    from paper_2603_03310_amd.runner import Decoder
    Hq, Hkv = HEADS[dtype, d]
    in_place = norms != (1, 1)
    rot, adjacent = PAIRS[pairs](d)
    size_of = 2 if dtype == "bf16" else 4
    assert (2 * T * (Hq + Hkv) * d * size_of > 160 << 20) == (T > 8000)
    g = torch.Generator(device="cuda:0")
    g.manual_seed(T + d)
    rows = torch.empty((T, Hq + 2 * Hkv, d), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32,
                       device="cuda:0").normal_(generator=g)
    rows *= torch.exp(torch.randn((T, 1, 1), generator=g, device="cuda:0")).to(rows.dtype)
    before = rows.clone()
    q, k = rows[:, :Hq], rows[:, Hq:Hq + Hkv]
    outs = (q, k) if in_place else tuple(torch.full(x.shape, -7.0, dtype=x.dtype, device="cuda:0") for x in (q, k))
    prm, gains = params(torch, np.random.default_rng(T), d, rot, adjacent, norms)
    starts = np.array([0, 1, 1, 900, 901, T - 70, T - 6])         # one of no rows; 6 of no request
    ctx = np.array([131000, 3, 0, 5, 16384, 77])
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    with Decoder(**config(Hq, Hkv, d, dtype, max_blocks_per_seq=8200)) as dec:
        dec.rotate(6, prm, q, k, *outs, starts=i32(starts), ctx_lens=i32(ctx))
        torch.cuda.synchronize()
        assert dec.device_status() == 0
    at, bad = OR.positions(T, starts, ctx, 8200 * 16)
    assert not bad and (at[-6:] == -1).all()
    pos = torch.tensor(at, device="cuda:0")
    for got, x, gain in ((outs[0], before[:, :Hq], gains[0]), (outs[1], before[:, Hq:Hq + Hkv], gains[1])):
        ref, size = formula(torch, x, pos, gain, freqs(rot), 1e-5, rot, adjacent)
        some = [0, 900, T - 7]
        want, most = OR.norm_rope(x[some].double().cpu().numpy(), at[some], gain, freqs(rot), 1e-5, rot, adjacent)
        assert np.allclose(ref[some].cpu().numpy(), want, rtol=1e-9, atol=1e-12)
        assert np.allclose(size[some].cpu().numpy(), most, rtol=1e-9, atol=1e-12)
        # The bound of tests/test_gpu_rotate.py.
        room = 17 * U32 * size + (BF16_HALF if dtype == "bf16" else U32) * ref.abs() + 1e-37
        err = (got.double() - ref).abs()[:T - 6]
        assert (err <= room[:T - 6]).all().item(), float((err / room[:T - 6]).max())
        assert torch.equal(got[T - 6:], x[T - 6:] if in_place else torch.full_like(x[T - 6:], -7.0))
    assert torch.equal(rows[:, Hq + Hkv:], before[:, Hq + Hkv:])
    if not in_place:
        assert torch.equal(rows, before)


@pytest.mark.parametrize("pairs", ["halves", "adjacent"])
def test_large_rows_of_few_steps(torch_cuda, pairs):
    """Three and four steps a row (16 + 4 heads of 64, 8 + 8 of 128), past the caches."""
    torch = torch_cuda
    from paper_2603_03310_amd.runner import Decoder
    for Hq, Hkv, d in ((16, 4, 64), (8, 8, 128)):
        rot, adjacent = PAIRS[pairs](d)
        T = (180 * 10**6) // (4 * (Hq + Hkv) * d)
        g = torch.Generator(device="cuda:0")
        g.manual_seed(T)
        q, k = (torch.empty((T, h, d), dtype=torch.bfloat16, device="cuda:0").normal_(generator=g) for h in (Hq, Hkv))
        outs = tuple(torch.empty_like(x) for x in (q, k))
        prm, gains = params(torch, np.random.default_rng(T), d, rot, adjacent, (1, 1))
        starts = torch.tensor([0, T // 3, T], dtype=torch.int32, device="cuda:0")
        with Decoder(**config(Hq, Hkv, d)) as dec:
            dec.rotate(2, prm, q, k, *outs, starts=starts)
            torch.cuda.synchronize()
            assert dec.device_status() == 0
        pos = torch.arange(T, device="cuda:0")
        pos[T // 3:] -= T // 3
        for got, x, gain in zip(outs, (q, k), gains):
            ref, size = formula(torch, x, pos, gain, freqs(rot), 1e-5, rot, adjacent)
            assert ((got.double() - ref).abs() <= 17 * U32 * size + BF16_HALF * ref.abs() + 1e-37).all().item()
