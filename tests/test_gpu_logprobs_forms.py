"""ent_token_logprobs in the forms that large calls take: bf16 rows that are read without a
place in the caches (more than 218 MB), and rows of some length to a wave each (2048 rows and
more of up to 32 KB on 256 CUs), with ties, masks, rows without a distribution, unaligned rows,
and more candidates than a wave ranks at once.  A sample of rows against the oracle."""
import numpy as np
import pytest

import tests.test_gpu_logprobs as L
from tests.prompt_data import U32
from tests.test_gpu_parity import torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu


def wave_bounds(lp, h, V):
    """tests/test_gpu_logprobs.py's, with the V / 64 terms that a lone wave's thread sums."""
    n, top = V / 64 + 80, np.log(V)
    return U32 * (n + 8 * (np.abs(lp) + top)), U32 * ((n + 20) * (1 + h) + 8 * top)


def logits(torch, T, V, dtype, pad, first, threads):
    """Rows V + pad apart from element `first` on, the first of them (`threads` to a row) special."""
    g = torch.Generator(device="cuda:0")
    g.manual_seed(T + V + pad)
    buf = torch.empty(first + T * (V + pad), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32,
                      device="cuda:0").normal_(0.0, 3.0, generator=g)
    z = buf[first:].view(T, V + pad)[:, :V]
    at = torch.arange(V, device="cuda:0")
    noise = torch.rand(V, generator=g, device="cuda:0")
    place = at // (4 if dtype == "f32" else 8) % threads
    ninf = float("-inf")
    z[0] = 2.5
    z[1] = torch.randint(0, 3, (V,), generator=g, device="cuda:0").to(z.dtype)
    z[2] = ninf
    z[2, [V - 1, 17, 300]] = torch.tensor([1.0, 1.0, -3.0], device="cuda:0").to(z.dtype)
    z[3], z[4] = at / 64, -at / 64
    z[5] = ninf
    z[6, V // 3] = float("nan")
    z[7, V - 2] = float("inf")
    z[8, V // 3:] = ninf
    z[9] = -3.0e38 if dtype == "f32" else -3.0e4
    z[10] = torch.where(place < 31, 20.0, 0.0) + noise             # 31 threads hold the largest
    z[11] = torch.where(place == 5, 20.0, 0.0) + noise             # one does
    z[12] = torch.where(at % 2 == 0, 0.0, -0.0)
    z[13, :40] = 30.0
    z[14, -40:] = 30.0
    z[15] = at % 2048
    return z


def check(torch, z, n, every, temp=None):
    T, V = z.shape
    rng = np.random.default_rng(n)
    tokens = rng.integers(0, V, T)
    sample = np.unique(np.concatenate([np.arange(20), np.arange(0, T, every), [T - 2, T - 1]]))
    tokens[sample[30]], tokens[T - 1], tokens[13] = -1, V, 0
    got = L.run(torch, z, tokens, n, temp)
    where = torch.tensor(sample, device="cuda:0")
    L.check(z[where], [x[sample] for x in got[:4]] + [got[4]], tokens[sample], n, None if temp is None else temp[sample])


@pytest.mark.parametrize("n,temps", [(0, False), (1, True), (5, False), (32, False)])
@pytest.mark.parametrize("pad,first", [(0, 0), (3, 5)])
def test_bf16_rows_past_the_caches(torch_cuda, pad, first, n, temps):
    torch = torch_cuda
    T, V = 1100, 100003
    assert 2 * T * V > 208 << 20
    z = logits(torch, T, V, "bf16", pad, first, 256)
    check(torch, z, n, 40, np.random.default_rng(1).uniform(0.3, 3.0, T) if temps else None)


@pytest.mark.parametrize("n,temps", [(0, False), (1, True), (20, False), (32, True)])
@pytest.mark.parametrize("V,dtype,pad,first", [(8000, "f32", 0, 0), (8191, "f32", 3, 1), (5000, "f32", 1, 2),
                                               (16000, "bf16", 0, 0), (16383, "bf16", 2, 5), (8192, "f32", 0, 0)])
def test_rows_to_a_wave_each(torch_cuda, monkeypatch, V, dtype, pad, first, n, temps):
    torch = torch_cuda
    monkeypatch.setattr(L, "bounds", wave_bounds)
    T = 8 * torch.cuda.get_device_properties(0).multi_processor_count + 5
    assert V * (2 if dtype == "bf16" else 4) <= 32 << 10
    z = logits(torch, T, V, dtype, pad, first, 64)
    check(torch, z, n, 7, np.random.default_rng(2).uniform(0.3, 3.0, T) if temps else None)
