"""Inputs and error bounds shared by the GPU tests of the prompt and 8-bit operators."""
import numpy as np

BF16_HALF = 2.0 ** -8       # half a step of bf16, relative to the value
U32 = 2.0 ** -24            # and of float32


def config(Hq, Hkv, d, dtype="bf16", **kw):
    return dict(dict(max_batch=64, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=d,
                     max_blocks_per_seq=64, num_pool_blocks=256, kv_dtype=int(dtype == "bf16"),
                     scale=1.0 / d ** 0.5), **kw)


def to_dev(torch, x, dtype="bf16"):
    """A float64 array on the GPU in the cache's type, and the values it then has."""
    t = torch.tensor(np.ascontiguousarray(x), device="cuda:0").to(
        torch.bfloat16 if dtype == "bf16" else torch.float32)
    return t, t.double().cpu().numpy()


def host(t):
    return t.double().cpu().numpy()


def attention_bound(out, mass, span, d, n, dtype):
    """How far an output may be from the exact one: weights (bf16: half a step each) and
    the output's own rounding; scores, a sum of d products in float32, move a weight by
    twice their error; the sums over n keys."""
    ds = (2 * (d + 8) * U32 * span + 2.0 ** -20)[..., None]
    if dtype == "bf16":
        return 1.01 * BF16_HALF * (mass + np.abs(out)) + (ds + 4 * n * U32) * mass
    return U32 * np.abs(out) + (ds + 4 * n * U32) * mass


def lse_bound(lse, span, d, n):
    return (d + 8) * U32 * span + 2 * n * U32 + 2.0 ** -20 + 4 * U32 * np.abs(lse)
