"""Decode attention over tokens whose key, value or query is not finite, in all three
forms (bf16, fp32, 8-bit cache), with the kept blocks in one piece and cut between waves
and workgroups: a NaN shows in every output that it enters and in no other, wherever the
segments are cut, and a score of minus infinity weighs nothing."""
import math

import pytest

from tests.test_gpu_parity import torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

# Tokens of each sequence; the one that is spoiled is sequence 0's.
BATCHES = {"one_block": [9], "few": [161, 40, 3], "cut": [2049, 17], "pieces": [16401],
           "many": [49] + [30] * 60}


def _program(torch, form, d, lens, seed=1):
    """Inputs of one call, heads 8 / 2, every block kept, blocks one behind the other."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    B, nbs = len(lens), [-(-n // 16) for n in lens]
    maxb, P = max(nbs), sum(nbs)
    i32 = dict(dtype=torch.int32, device="cuda")
    tab = torch.full((B, maxb), -1, **i32)
    at = 0
    for b, nb in enumerate(nbs):
        tab[b, :nb] = torch.arange(at, at + nb, **i32)
        at += nb
    edt = torch.float32 if form == "f32" else torch.bfloat16
    x = dict(q=normal(B, 8, d).to(edt), k=normal(P, 2, 16, d), v=normal(P, 2, d, 16))
    if form == "q8":
        x["k"], x["v"] = (t.clamp(-8, 8).mul(50).to(torch.float8_e4m3fn).view(torch.uint8)
                          for t in (x["k"], x["v"]))
    else:
        x["k"], x["v"] = x["k"].to(edt), x["v"].to(edt)
    x.update(tab=tab, lens=torch.tensor(lens, **i32), nk=torch.tensor(nbs, **i32),
             kept=torch.arange(maxb, **i32).expand(B, maxb).contiguous(),
             scale=torch.full((P, 2), 0.02, device="cuda"))
    return x


def _decode(torch, form, d, x):
    from paper_2603_03310_amd import ent
    from paper_2603_03310_amd.runner import Decoder
    B, maxb = x["tab"].shape
    out = torch.full((B, 8, d), -7.0, device="cuda")
    lse = torch.full((B, 8), -7.0, device="cuda")
    with Decoder(max_batch=B, num_q_heads=8, num_kv_heads=2, head_dim=d, max_blocks_per_seq=maxb,
                 num_pool_blocks=x["k"].shape[0], kv_dtype=int(form != "f32"),
                 scale=1.0 / math.sqrt(d)) as dec:
        tail = (x["tab"], x["lens"], x["kept"], x["nk"], out, lse)
        if form == "q8":
            ent.ent_sparse_paged_decode_q8(dec.ctx, B, x["q"], x["k"], x["v"], x["scale"], x["scale"], *tail)
        else:
            ent.ent_sparse_paged_decode(dec.ctx, B, x["q"], x["k"], x["v"], *tail)
        assert dec.device_status() == 0
    return out, lse


def _tokens(lens):
    """Tokens of sequence 0 to spoil: its first, one inside, its last."""
    return sorted({0, lens[0] // 2, lens[0] - 1})


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", BATCHES.values(), ids=BATCHES.keys())
@pytest.mark.parametrize("form", ["bf16", "f32", "q8"])
def test_nan_shows_where_it_enters(torch_cuda, form, lens, d):
    torch = torch_cuda
    nan = 0x7f if form == "q8" else math.nan
    x = _program(torch, form, d, lens)
    out, lse = _decode(torch, form, d, x)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()

    def same(o, l, hit_o, hit_l):
        assert torch.isnan(o[hit_o]).all() and torch.isnan(l[hit_l]).all()
        assert torch.equal(o[~hit_o], out[~hit_o]) and torch.equal(l[~hit_l], lse[~hit_l])

    none_o, none_l = torch.zeros_like(out, dtype=torch.bool), torch.zeros_like(lse, dtype=torch.bool)
    for t in _tokens(lens):
        # A key of KV head 1: query heads 4 to 7 of sequence 0.
        k = x["k"].clone()
        k[t // 16, 1, t % 16, 5] = nan
        hit_o, hit_l = none_o.clone(), none_l.clone()
        hit_o[0, 4:], hit_l[0, 4:] = True, True
        same(*_decode(torch, form, d, dict(x, k=k)), hit_o, hit_l)
        # A value: its dim alone, and not the sums.
        v = x["v"].clone()
        v[t // 16, 1, 7, t % 16] = nan
        hit_o = none_o.clone()
        hit_o[0, 4:, 7] = True
        same(*_decode(torch, form, d, dict(x, v=v)), hit_o, none_l)
    # A query: its head alone.
    q = x["q"].clone()
    q[0, 3, 2] = math.nan
    hit_o, hit_l = none_o.clone(), none_l.clone()
    hit_o[0, 3], hit_l[0, 3] = True, True
    same(*_decode(torch, form, d, dict(x, q=q)), hit_o, hit_l)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[161, 40, 3], [2049, 17], [16401]], ids=str)
@pytest.mark.parametrize("form", ["bf16", "f32"])
def test_a_score_of_minus_infinity_weighs_nothing(torch_cuda, form, lens, d):
    """An infinite key: heads whose score it makes -inf attend over the other tokens, heads
    whose score it makes +inf have no finite answer.  The last token has a block of its own."""
    torch = torch_cuda
    x = _program(torch, form, d, lens)
    x["q"][:, ::2, 5] = -1.0
    x["q"][:, 1::2, 5] = 1.0
    scale = float(torch.tensor(1.0 / math.sqrt(d)).float())
    for t in _tokens(lens):
        k = x["k"].clone()
        k[t // 16, :, t % 16, 5] = math.inf
        out, lse = _decode(torch, form, d, dict(x, k=k))
        nb, n = -(-lens[0] // 16), lens[0]
        keys = x["k"][:nb].double().permute(1, 0, 2, 3).reshape(2, -1, d)[:, :n].contiguous()
        vals = x["v"][:nb].double().permute(1, 0, 3, 2).reshape(2, -1, d)[:, :n].contiguous()
        s = scale * torch.matmul(x["q"][0].double().view(2, 4, d), keys.transpose(1, 2).contiguous())
        s[:, :, t] = -math.inf
        ref = torch.matmul(torch.softmax(s, 2), vals).reshape(8, d)
        # Weights of 16 bits at least (fp32: 24) times values of at most 6, and 32-bit sums.
        tol = 6 * 2.0 ** -17 + 1e-5 if form == "bf16" else 1e-5
        assert float((out[0, ::2].double() - ref[::2]).abs().max()) <= tol
        want = torch.logsumexp(s, 2).reshape(8)
        assert float((lse[0, ::2].double() - want[::2]).abs().max()) <= 1e-5 * max(1.0, float(want.abs().max()))
        assert not torch.isfinite(out[0, 1::2]).any()
