"""Requests through the library as a serving program has it: plan, store and
attention of packed prompts, then decode steps that grow the tables, decode and
append, with a bf16 and with an 8-bit cache; every stage against the oracle on
the cache as it then is.  The whole of it captured in a graph and replayed
equals the eager calls bit for bit."""
import numpy as np
import pytest

from oracle import attention as OA
from oracle import layout as OL
from oracle import prompt as OP
from tests.prompt_data import attention_bound, config, host, to_dev
from tests.test_gpu_parity import torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

HQ, H, D, V = 8, 2, 128, 700
LENS = [33, 0, 1, 160, 16, 250, 15]
STEPS = 4


def _i32(torch, x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda:0")


class Program:
    """Buffers of a program, and its two calls' worth of work."""

    def __init__(self, torch, q8, seed=0):
        from paper_2603_03310_amd.runner import Decoder
        rng = np.random.default_rng(seed)
        self.torch, self.q8, self.B = torch, q8, len(LENS)
        self.P, self.maxb, self.T = 60, 20, sum(LENS) + 21
        B, P = self.B, self.P
        f = lambda *s: torch.zeros(*s, device="cuda:0")
        self.dec = Decoder(**config(HQ, H, D, max_batch=B, max_blocks_per_seq=self.maxb,
                                    num_pool_blocks=P, vocab=V, log_v=float(np.log(V)), h_target=2.0,
                                    h_min=2.0))
        edt = torch.uint8 if q8 else torch.bfloat16
        self.kc = torch.randint(0, 255, (P, H, 16, D), device="cuda:0").to(edt)
        self.vc = torch.randint(0, 255, (P, H, D, 16), device="cuda:0").to(edt)
        self.sc = [f(P, H) + 7.0, f(P, H) + 7.0] if q8 else [None, None]
        self.ksum = f(P, H, D)
        self.tab = _i32(torch, np.full((B, self.maxb), -1))
        self.ids = _i32(torch, rng.permutation(P))
        self.free, self.starts = _i32(torch, [0, P]), _i32(torch, [0] * (B + 1))
        self.n_new, self.ones, self.lens = _i32(torch, LENS), _i32(torch, [1] * B), _i32(torch, [0] * B)
        self.new_lens = _i32(torch, [0] * B)
        self.slots = torch.zeros(self.T, dtype=torch.int64, device="cuda:0")
        self.dslots = torch.zeros(B, dtype=torch.int64, device="cuda:0")
        self.dstarts = _i32(torch, [0] * (B + 1))
        self.rows, _ = to_dev(torch, rng.normal(size=(self.T, HQ + 2 * H, D)))
        self.pout = torch.full((self.T, HQ, D), -7.0, dtype=torch.bfloat16, device="cuda:0")
        self.q, _ = to_dev(torch, rng.normal(size=(STEPS, B, HQ, D)))
        self.kn, _ = to_dev(torch, rng.normal(size=(STEPS, B, H, D)) * 2)
        self.vn, _ = to_dev(torch, rng.normal(size=(STEPS, B, H, D)) * 2)
        self.logits = torch.tensor(rng.normal(size=(STEPS, B, V)) * 2, device="cuda:0").float()
        self.u = torch.tensor(rng.random((STEPS, B)), device="cuda:0").float()
        self.state = dict(h_prev=f(B) + float("nan"), tau=f(B), temp=f(B) + 1.0)
        self.h, self.tu, self.rs = f(B), f(B), f(B, 1, 2)
        self.kept, self.nk = _i32(torch, np.full((B, self.maxb), -1)), _i32(torch, [0] * B)
        self.out, self.tok = f(STEPS, B, HQ, D), _i32(torch, np.zeros((STEPS, B)))

    def prompts(self):
        d = self.dec
        q, k, v = self.rows[:, :HQ], self.rows[:, HQ:HQ + H], self.rows[:, HQ + H:]
        d.plan(self.B, self.n_new, self.lens, self.tab, self.ids, self.free, self.starts, self.slots,
               self.new_lens)
        d.store(k, v, self.slots, self.kc, self.vc, self.ksum, *self.sc)
        d.prompt(self.B, q, k, v, self.starts, self.pout)
        self.lens.copy_(self.new_lens)

    def step(self, i):
        d = self.dec
        d.plan(self.B, self.ones, self.lens, self.tab, self.ids, self.free, self.dstarts, self.dslots)
        d.step(self.B, logits=self.logits[i], q=self.q[i], k_cache=self.kc, v_cache=self.vc,
               block_tables=self.tab, ctx_lens=self.lens, ksum=self.ksum, uniforms=self.u[i], h=self.h,
               temp_used=self.tu, row_stats=self.rs, kept=self.kept, n_kept=self.nk, out=self.out[i],
               tokens=self.tok[i], k_scale=self.sc[0], v_scale=self.sc[1], **self.state)
        d.append(self.B, self.kn[i], self.vn[i], self.tab, self.lens, self.kc, self.vc, self.ksum,
                 k_scale=self.sc[0], v_scale=self.sc[1])

    def tensors(self):
        return [t for v in vars(self).values() for t in (v if isinstance(v, list) else
                v.values() if isinstance(v, dict) else [v]) if self.torch.is_tensor(t)]

    def cache(self):
        """Keys and values that the cache holds, float64."""
        if not self.q8:
            return host(self.kc), host(self.vc)
        t = OP.e4m3_values()
        return tuple(t[c.cpu().numpy()] * host(s)[:, :, None, None]
                     for c, s in zip((self.kc, self.vc), self.sc))


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_prompts_then_steps(torch_cuda, q8):
    torch = torch_cuda
    p = Program(torch, q8)
    scale = float(np.float32(p.dec.cfg.scale))
    tab0, ids = p.tab.cpu().numpy(), p.ids.cpu().numpy()
    p.prompts()
    want = OP.plan(LENS, [0] * p.B, tab0, ids, [0, p.P], p.T, p.P)
    for got, ref in zip((p.tab, p.starts, p.slots, p.new_lens, p.free), want):
        assert np.array_equal(got.cpu().numpy(), ref)
    x = host(p.rows)
    q, k, v = x[:, :HQ], x[:, HQ:HQ + H], x[:, HQ + H:]
    E = sum(LENS)
    ref, _, mass, span = OP.attention(q, k, v, want[1], scale)
    assert (np.abs(host(p.pout) - ref)[:E] <= attention_bound(ref, mass, span, D, 250, "bf16")[:E]).all()
    # The cache holds the prompts: exactly, or within half a step of e4m3 (2^-4 of the value,
    # or half the smallest step of the tile's scale, 2^-10).
    K, W = p.cache()
    lens = list(LENS)
    for b, n in enumerate(lens):
        Kb, Vb = OL.gather_sequence(K, W, want[0][b], n, 16)
        a = want[1][b]
        for got, src, sc in ((Kb, k, p.sc[0]), (Vb, v, p.sc[1])):
            err = np.abs(got - src[a:a + n])
            if q8 and n:
                s = host(sc)[want[0][b, :-(-n // 16)]].repeat(16, 0)[:n, :, None]
                assert (err <= 2.0 ** -4 * np.abs(src[a:a + n]) + 2.0 ** -10 * s).all()
            else:
                assert (err == 0).all()
    tab, r = want[0], want[4]
    for i in range(STEPS):
        ctx = np.array(lens)
        p.step(i)
        tab, _, sl, _, r, f = OP.plan([1] * p.B, ctx, tab, ids, r, p.B, p.P)
        assert f == 0 and np.array_equal(p.tab.cpu().numpy(), tab)
        assert np.array_equal(p.dslots.cpu().numpy(), sl)
        kept, nk = p.kept.cpu().numpy(), p.nk.cpu().numpy()
        o, qi = host(p.out[i]), host(p.q[i])
        for b, n in enumerate(lens):
            Kb, Vb = OL.gather_sequence(K, W, tab[b], n, 16)
            ref, _ = OA.sparse_decode(qi[b], Kb, Vb, kept[b, :nk[b]], 16, scale)
            assert nk[b] >= min(4, -(-n // 16)) and np.abs(o[b] - ref).max() <= 2e-5
        lens = [n + 1 for n in lens]
        assert p.lens.cpu().tolist() == lens
        K, W = p.cache()
        means = host(p.ksum)
        for b, n in enumerate(lens):
            j, m = (n - 1) // 16, (n - 1) % 16 + 1
            assert np.allclose(means[tab[b, j]], K[tab[b, j], :, :m].mean(1), rtol=1e-5, atol=1e-6)
    assert p.dec.device_status() == 0
    p.dec.close()


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_graph_replays_equal_eager(torch_cuda, q8):
    torch = torch_cuda

    def work(p):
        p.prompts()
        for i in range(STEPS):
            p.step(i)

    p = Program(torch, q8)
    saved = [t.clone() for t in p.tensors()]

    def restore():
        for t, s in zip(p.tensors(), saved):
            t.copy_(s)
        torch.cuda.synchronize()

    work(p)
    torch.cuda.synchronize()
    want = [t.clone() for t in p.tensors()]
    restore()
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        work(p)
    for _ in range(3):
        restore()
        p.pout.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(p.tensors(), want):
            if a is p.pout:
                a, b = a[:sum(LENS)], b[:sum(LENS)]
            assert torch.equal(torch.nan_to_num(a.double()), torch.nan_to_num(b.double()))
        assert torch.isfinite(p.out).all().item()
    assert p.dec.device_status() == 0
    p.dec.close()
