"""A plan whose free range lies outside its list serves no request, those neither that
need no new block."""
import numpy as np
import pytest

from oracle import prompt as OP
from tests.test_gpu_parity import torch_cuda  # noqa: F401

# Requests whose tokens fit the block that they have begun, among others.
N_NEW, CTX = [1, 0, 3, 20, 1], [3, 16, 29, 5, 15]
TABLES = np.array([[4, -1, -1], [5, -1, -1], [6, 7, -1], [8, -1, -1], [9, -1, -1]])
RANGES = [[0, 9], [-1, 8], [6, 5], [-3, -1], [9, 9], [0, 1 << 30], [1 << 30, 0]]


@pytest.mark.parametrize("r", RANGES, ids=str)
def test_the_oracle_serves_nobody(r):
    tab, starts, slots, lens, free, flags = OP.plan(N_NEW, CTX, TABLES, list(range(8)), r, 32, 12)
    assert np.array_equal(tab, TABLES) and (starts == 0).all() and (slots == -1).all()
    assert list(lens) == CTX and list(free) == r
    assert flags == OP.BAD_TABLE | OP.CACHE_FULL


def test_the_oracle_serves_those_without_need_of_a_block():
    """... where the list is good and merely empty."""
    _, starts, slots, lens, _, flags = OP.plan([1, 3], [3, 29], TABLES[[0, 2]], [], [0, 0], 32, 12)
    assert list(starts) == [0, 1, 4] and list(lens) == [4, 32] and flags == 0
    assert list(slots[:5]) == [4 * 16 + 3, 7 * 16 + 13, 7 * 16 + 14, 7 * 16 + 15, -1]


@pytest.mark.gpu
@pytest.mark.parametrize("r", RANGES, ids=str)
def test_the_plan_serves_nobody(torch_cuda, r):
    torch = torch_cuda
    from paper_2603_03310_amd.runner import Decoder
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda:0")  # noqa: E731
    tab, free, starts, lens = i32(TABLES), i32(r), i32([-7] * 6), i32([-7] * 5)
    slots = torch.full((32,), -7, dtype=torch.int64, device="cuda:0")
    with Decoder(max_batch=5, num_q_heads=8, num_kv_heads=8, head_dim=64, max_blocks_per_seq=3,
                 num_pool_blocks=12) as dec:
        dec.plan(5, i32(N_NEW), i32(CTX), tab, i32(range(8)), free, starts, slots, lens)
        torch.cuda.synchronize()
        assert dec.device_status() == OP.BAD_TABLE | OP.CACHE_FULL
        assert (starts == 0).all() and (slots == -1).all()
        assert lens.tolist() == CTX and free.tolist() == r and tab.tolist() == TABLES.tolist()
        # The list put right: the same call serves them.
        free = i32([0, 8])
        dec.plan(5, i32(N_NEW), i32(CTX), tab, i32(range(8)), free, starts, slots, lens)
        torch.cuda.synchronize()
        assert dec.device_status() == 0
    want = OP.plan(N_NEW, CTX, TABLES, list(range(8)), [0, 8], 32, 12)
    for got, ref in zip((tab, starts, slots, lens, free), want):
        assert np.array_equal(got.cpu().numpy(), ref)
