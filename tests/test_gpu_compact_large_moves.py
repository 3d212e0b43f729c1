"""ent_cache_compact on both sides of the traffic from which on moves take no places in the
caches (some 150 MB read and written): every cache type, tiles of 2 KB to 64 KB, bit for bit."""
import numpy as np
import pytest

from tests.test_gpu_pages import Pool, decoder
from tests.test_gpu_parity import torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("large", [False, True])
@pytest.mark.parametrize("kind,H,D", [("bf16", 8, 128), ("q8", 8, 128), ("f32", 8, 128), ("bf16", 6, 128),
                                      ("bf16", 1, 64), ("q8", 3, 64)])
def test_moves(torch_cuda, kind, H, D, large):
    tile = H * D * 16 * {"bf16": 2, "q8": 1, "f32": 4}[kind]
    used = int((220 if large else 100) * 1e6 / (2 * tile))       # about half of them move, in a pool of twice as many
    rng = np.random.default_rng(used)
    R = 40
    nb = np.full(R, used // R)
    lens = nb * 16 - rng.integers(0, 16, R)
    p = Pool(torch_cuda, lens, R, 2 * used, int(nb.max()), kind, H, D, seed=1)
    p.upload()
    before = p.tables.copy()
    with decoder(p) as dec:
        p.both(dec, "compact", flags=0)
    moved = sum(int((before[r, :nb[r]] != p.tables[r, :nb[r]]).sum()) for r in range(R))
    assert (moved * 4 * tile > 151 * 10**6) == large and moved * 4 * tile > 60 * 10**6
