"""ent_cache_compact of no sequences: every block is free."""
import numpy as np
import pytest

from tests.test_gpu_pages import Pool, decoder
from tests.test_gpu_parity import torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "q8"])
@pytest.mark.parametrize("P,pad", [(1, 0), (64, 3), (5000, 0)])
def test_the_whole_pool_is_free(torch_cuda, kind, P, pad):
    p = Pool(torch_cuda, [], 0, P, 4, kind, 1, 64, seed=P, pad=pad)
    p.ids[:], p.free = -9, [7, -3]
    p.shared[:] = np.arange(P) % 5 - 2
    p.upload()
    with decoder(p) as dec:
        p.both(dec, "compact", flags=0)
        assert p.count == 0 and p.free == [pad, P + pad] and (p.shared == 0).all()
        p.d["free"].fill_(-5)
        p.both(dec, "compact", shared=False, flags=0)


def test_arrays_left_out(torch_cuda):
    from paper_2603_03310_amd import ent
    torch = torch_cuda
    p = Pool(torch, [], 0, 40, 4, seed=1)
    p.upload()
    d = p.d
    k, v, ksum, _ = p.caches()
    with decoder(p) as dec:
        def call(ids=d["ids"], free=d["free"], k=k, shared=d["shared"], n_ids=40):
            ent.ent_cache_compact(dec.ctx, 0, None, None, shared, ids, n_ids, free, k, v, None, None, ksum, p.used)

        for kw in (dict(ids=None), dict(free=None), dict(k=None), dict(k=k.data_ptr() + 8), dict(n_ids=39),
                   dict(ids=None, free=None)):
            with pytest.raises(ent.EntError) as e:
                call(**kw)
            assert e.value.code == ent.ENT_E_INVAL, kw
        torch.cuda.synchronize()
        p.same()
        ent.ent_cache_compact(dec.ctx, 0, *[None] * 4, 40, *[None] * 6)      # no array at all: nothing
        torch.cuda.synchronize()
        p.same()
        call()                                                              # neither tables nor lengths
        torch.cuda.synchronize()
        assert p.oracle("compact") == 0
        p.same()
        assert int(p.used[0]) == 0
