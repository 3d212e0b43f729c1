"""Requests from their prompts to their end, as a serving program has them: queries and keys
normalised and turned in their projection's rows, plan, store, attention, log probabilities of
the prompt; then samples of each request (forks), decode steps that grow, decode, append and
score their tokens, some samples ending, the pool compacted, and more steps.  Every stage
against the oracle on the cache as it then is, with a bf16 and an 8-bit cache; and the whole of
it captured in a graph and replayed equals the eager calls bit for bit."""
import numpy as np
import pytest

from oracle import attention as OA
from oracle import layout as OL
from oracle import logprobs as OP
from oracle import pages as OG
from oracle import prompt as OPr
from oracle import rotate as OR
from tests.prompt_data import attention_bound, config, host, to_dev
from tests.test_gpu_logprobs import bounds as logprob_bounds
from tests.test_gpu_parity import torch_cuda  # noqa: F401
from tests.test_gpu_rotate import bound as rotate_bound
from tests.test_gpu_rotate import freqs

pytestmark = pytest.mark.gpu

HQ, H, D, V, TOP = 8, 2, 128, 700, 4
LENS = [33, 160, 16, 47]                       # prompts, in rows 0 .. 3
SRC, DST = [1, 0, 3, 1, 2, 1], [4, 5, 6, 7, 8, 9]
ENDS = [9, 8, 7]                               # the last rows, so rows 0 .. 6 stay
STEPS = [10, 10, 7, 7]                         # sequences of each step
EPS = 1e-6


class Program:
    def __init__(self, torch, q8, seed=0):
        from paper_2603_03310_amd import ent
        from paper_2603_03310_amd.runner import Decoder
        rng = np.random.default_rng(seed)
        self.torch, self.q8 = torch, q8
        R = self.R = len(LENS) + len(DST)
        P = self.P = 70
        self.maxb, self.T, B = 14, sum(LENS) + 9, len(LENS)
        f = lambda *s: torch.zeros(*s, device="cuda:0")  # noqa: E731
        i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda:0")  # noqa: E731
        self.dec = Decoder(**config(HQ, H, D, max_batch=R, max_blocks_per_seq=self.maxb, num_pool_blocks=P,
                                    vocab=V, log_v=float(np.log(V)), h_target=2.0, h_min=2.0))
        self.gains = [1 + 0.2 * rng.normal(size=D).astype(np.float32) for _ in range(2)]
        dev = [torch.tensor(x, device="cuda:0") for x in self.gains + [freqs(D)]]
        self.prm = ent.make_qk_params(*dev, EPS, D)
        edt = torch.uint8 if q8 else torch.bfloat16
        self.kc = torch.zeros((P, H, 16, D), device="cuda:0").to(edt)
        self.vc = torch.zeros((P, H, D, 16), device="cuda:0").to(edt)
        self.sc = [f(P, H) + 1.0, f(P, H) + 1.0] if q8 else [None, None]
        self.ksum, self.shared = f(P, H, D), i32(np.zeros(P))
        self.tab, self.lens = i32(np.full((R, self.maxb), -1)), i32([0] * R)
        self.ids, self.free = i32(rng.permutation(P)), i32([0, P])
        self.n_new, self.ones = i32(LENS), i32([1] * R)
        self.new_lens, self.starts = i32([0] * B), i32([0] * (B + 1))
        self.slots = torch.zeros(self.T, dtype=torch.int64, device="cuda:0")
        self.dslots = torch.zeros(R, dtype=torch.int64, device="cuda:0")
        self.dstarts = i32([0] * (R + 1))
        self.rows, self.rows0 = to_dev(torch, rng.normal(size=(self.T, HQ + 2 * H, D)))
        self.pout = torch.full((self.T, HQ, D), -7.0, dtype=torch.bfloat16, device="cuda:0")
        self.step_rows, self.step0 = to_dev(torch, rng.normal(size=(len(STEPS), R, HQ + 2 * H, D)))
        self.q, self.kn, self.vn = ([torch.zeros((R, h, D), dtype=torch.bfloat16, device="cuda:0") for _ in STEPS]
                                    for h in (HQ, H, H))
        self.plogits = torch.tensor(rng.normal(size=(self.T, V)) * 2, device="cuda:0").to(torch.bfloat16)
        self.ptok = i32(np.where(np.arange(self.T) < sum(LENS), rng.integers(0, V, self.T), -1))
        self.logits = torch.tensor(rng.normal(size=(len(STEPS), R, V)) * 2, device="cuda:0").float()
        self.u = torch.tensor(rng.random((len(STEPS), R)), device="cuda:0").float()
        self.state = dict(h_prev=f(R) + float("nan"), tau=f(R), temp=f(R) + 1.0)
        self.h, self.tu, self.rs = f(R), f(R), f(R, 1, 2)
        self.kept, self.nk = i32(np.full((R, self.maxb), -1)), i32([0] * R)
        self.out, self.tok = f(len(STEPS), R, HQ, D), i32(np.zeros((len(STEPS), R)))
        n = self.T
        self.plp, self.ph, self.pids, self.ptop = f(n), f(n), i32(np.zeros((n, TOP))), f(n, TOP)
        self.lp, self.lh = f(len(STEPS), R), f(len(STEPS), R)
        self.src, self.dst, self.ends = i32(SRC), i32(DST), i32(ENDS)
        self.used = i32([0])

    def prompts(self):
        d, x, B = self.dec, self.rows, len(LENS)
        q, k, v = x[:, :HQ], x[:, HQ:HQ + H], x[:, HQ + H:]
        d.plan(B, self.n_new, self.lens[:B], self.tab, self.ids, self.free, self.starts, self.slots, self.new_lens)
        d.rotate(B, self.prm, q, k, q, k, starts=self.starts, ctx_lens=self.lens)
        d.store(k, v, self.slots, self.kc, self.vc, self.ksum, *self.sc)
        d.prompt(B, q, k, v, self.starts, self.pout)
        d.logprobs(self.plogits, self.ptok, self.plp, self.ph, self.pids, self.ptop)
        self.lens[:B].copy_(self.new_lens)

    def fork(self):
        self.dec.fork(self.src, self.dst, self.tab, self.lens, self.shared, self.ids, self.free, self.kc, self.vc,
                      self.ksum, *self.sc)

    def step(self, i):
        d, n = self.dec, STEPS[i]
        x = self.step_rows[i]
        d.plan(n, self.ones, self.lens, self.tab, self.ids, self.free, self.dstarts, self.dslots[:n])
        d.rotate(n, self.prm, x[:n, :HQ], x[:n, HQ:HQ + H], self.q[i][:n], self.kn[i][:n], ctx_lens=self.lens)
        self.vn[i].copy_(x[:, HQ + H:])
        d.step(n, logits=self.logits[i], q=self.q[i], k_cache=self.kc, v_cache=self.vc, block_tables=self.tab,
               ctx_lens=self.lens, ksum=self.ksum, uniforms=self.u[i], h=self.h, temp_used=self.tu,
               row_stats=self.rs, kept=self.kept, n_kept=self.nk, out=self.out[i], tokens=self.tok[i],
               k_scale=self.sc[0], v_scale=self.sc[1], **self.state)
        d.logprobs(self.logits[i][:n], self.tok[i][:n], self.lp[i][:n], self.lh[i][:n], temp=self.tu)
        d.append(n, self.kn[i], self.vn[i], self.tab, self.lens, self.kc, self.vc, self.ksum,
                 k_scale=self.sc[0], v_scale=self.sc[1])

    def end(self):
        self.dec.release(self.ends, self.tab, self.lens, self.ids, self.free, self.shared)
        self.dec.compact(self.tab, self.lens, self.ids, self.free, self.kc, self.vc, self.ksum, self.shared,
                         *self.sc, n_used=self.used)

    def work(self):
        self.prompts()
        self.fork()
        self.step(0)
        self.step(1)
        self.end()
        self.step(2)
        self.step(3)

    def tensors(self):
        return [t for v in vars(self).values() for t in (v if isinstance(v, list) else
                v.values() if isinstance(v, dict) else [v]) if self.torch.is_tensor(t)]

    def cache(self):
        if not self.q8:
            return host(self.kc), host(self.vc)
        t = OPr.e4m3_values()
        return tuple(t[c.cpu().numpy()] * host(s)[:, :, None, None] for c, s in zip((self.kc, self.vc), self.sc))


class Host:
    """What the program should hold: tables, lengths, counts, list, and every token's key and value."""

    def __init__(self, p):
        self.p = p
        self.tab, self.lens = p.tab.cpu().numpy().astype(int), np.zeros(p.R, int)
        self.shared, self.ids, self.free = np.zeros(p.P, int), p.ids.cpu().numpy().astype(int), [0, p.P]
        self.k = [np.zeros((0, H, D)) for _ in range(p.R)]
        self.v = [np.zeros((0, H, D)) for _ in range(p.R)]

    def plan(self, n, n_new):
        tab, starts, slots, lens, free, f = OPr.plan(n_new, self.lens[:n], self.tab[:n], self.ids, self.free, 10000,
                                                     self.p.P)
        assert f == 0
        self.tab[:n], self.free = tab, list(free)
        return starts, lens

    def same(self):
        p = self.p
        for name, want in (("tab", self.tab), ("lens", self.lens), ("shared", self.shared), ("ids", self.ids),
                           ("free", self.free)):
            assert np.array_equal(getattr(p, name).cpu().numpy(), np.asarray(want)), name
        K, W = p.cache()
        for b, n in enumerate(self.lens):
            kb, vb = OL.gather_sequence(K, W, self.tab[b], n, 16)
            for got, ref, sc in ((kb, self.k[b], p.sc[0]), (vb, self.v[b], p.sc[1])):
                err = np.abs(got - ref)
                if p.q8 and n:
                    # Half a step of e4m3, of the value or the smallest of its scale, and once
                    # more for each time that the tile's scale grew (twice at the most here).
                    s = host(sc)[self.tab[b, :-(-n // 16)]].repeat(16, 0)[:n, :, None]
                    assert (err <= 3 * (2.0 ** -4 * np.abs(ref) + 2.0 ** -10 * s)).all()
                else:
                    assert (err == 0).all()
        return K, W


def turned(p, x, pos, which):
    ref, size = OR.norm_rope(x, pos, p.gains[which], freqs(D), EPS, D, False)
    return ref, rotate_bound(ref, size, "bf16")


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_from_prompts_to_the_end(torch_cuda, q8):
    p = Program(torch_cuda, q8)
    w = Host(p)
    scale = float(np.float32(p.dec.cfg.scale))
    B, E = len(LENS), sum(LENS)
    p.prompts()
    starts, lens = w.plan(B, LENS)
    x = host(p.rows)
    pos, _ = OR.positions(p.T, starts, None, 1 << 20)
    for which, part in ((0, slice(0, HQ)), (1, slice(HQ, HQ + H))):
        ref, tol = turned(p, p.rows0[:, part], pos, which)
        assert (np.abs(x[:, part] - ref)[:E] <= tol[:E]).all()
        assert np.array_equal(x[E:], p.rows0[E:]) and np.array_equal(x[:, HQ + H:], p.rows0[:, HQ + H:])
    q, k, v = x[:, :HQ], x[:, HQ:HQ + H], x[:, HQ + H:]
    ref, _, mass, span = OPr.attention(q, k, v, starts, scale)
    assert (np.abs(host(p.pout) - ref)[:E] <= attention_bound(ref, mass, span, D, max(LENS), "bf16")[:E]).all()
    z = host(p.plogits)
    for t in range(E):
        r = OP.token_logprobs(z[t], int(p.ptok[t]), 1.0, TOP)
        b = logprob_bounds(r[3], r[1], V)
        assert abs(float(p.plp[t]) - r[0]) <= logprob_bounds(r[0], r[1], V)[0] and abs(float(p.ph[t]) - r[1]) <= b[1]
        assert np.array_equal(p.pids[t].cpu().numpy(), r[2]) and (np.abs(host(p.ptop[t]) - r[3]) <= b[0]).all()
    assert (p.plp[E:] == 0).all().item()
    for b in range(B):
        w.k[b], w.v[b] = k[starts[b]:starts[b + 1]], v[starts[b]:starts[b + 1]]
    w.lens[:B] = lens
    w.same()

    p.fork()
    assert OG.fork(SRC, DST, w.tab, w.lens, w.shared, w.ids, w.free, p.P) == 0
    for s, d in zip(SRC, DST):
        w.k[d], w.v[d] = w.k[s].copy(), w.v[s].copy()
    K, W = w.same()

    for i, n in enumerate(STEPS):
        if i == 2:
            p.end()
            assert OG.release(ENDS, w.tab, w.lens, w.shared, w.ids, w.free, p.P) == 0
            flags, used = OG.compact(w.tab, w.lens, w.shared, w.ids, w.free, p.P)
            assert flags == 0 and int(p.used[0]) == used
            for r in ENDS:
                w.k[r], w.v[r] = w.k[r][:0], w.v[r][:0]
            K, W = w.same()
        ctx = w.lens[:n].copy()
        p.step(i)
        w.plan(n, [1] * n)
        for which, part, got in ((0, slice(0, HQ), p.q[i]), (1, slice(HQ, HQ + H), p.kn[i])):
            ref, tol = turned(p, p.step0[i, :n, part], ctx, which)
            assert (np.abs(host(got)[:n] - ref) <= tol).all()
        kept, nk, o, qi = p.kept.cpu().numpy(), p.nk.cpu().numpy(), host(p.out[i]), host(p.q[i])
        z, temps = host(p.logits[i]), host(p.tu)
        for b in range(n):
            kb, vb = OL.gather_sequence(K, W, w.tab[b], ctx[b], 16)
            ref, _ = OA.sparse_decode(qi[b], kb, vb, kept[b, :nk[b]], 16, scale)
            assert nk[b] >= min(4, -(-ctx[b] // 16)) and np.abs(o[b] - ref).max() <= 2e-5
            r = OP.token_logprobs(z[b], int(p.tok[i, b]), temps[b], 0)
            tol = logprob_bounds(r[0], r[1], V)
            assert abs(float(p.lp[i, b]) - r[0]) <= tol[0] and abs(float(p.lh[i, b]) - r[1]) <= tol[1]
            w.k[b] = np.concatenate([w.k[b], host(p.kn[i])[None, b]])
            w.v[b] = np.concatenate([w.v[b], host(p.vn[i])[None, b]])
        w.lens[:n] += 1
        K, W = w.same()
    # All end: every block is free again.
    p.dec.release(p.torch.arange(p.R, dtype=p.torch.int32, device="cuda:0"), p.tab, p.lens, p.ids, p.free, p.shared)
    assert p.free.tolist() == [0, p.P] and sorted(p.ids.tolist()) == list(range(p.P)) and not p.shared.any().item()
    assert p.dec.device_status() == 0
    p.dec.close()


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_graph_replays_equal_eager(torch_cuda, q8):
    torch = torch_cuda
    p = Program(torch, q8)
    saved = [t.clone() for t in p.tensors()]

    def restore():
        for t, s in zip(p.tensors(), saved):
            t.copy_(s)
        torch.cuda.synchronize()

    p.work()
    torch.cuda.synchronize()
    want = [t.clone() for t in p.tensors()]
    restore()
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        p.work()
    for _ in range(3):
        restore()
        p.pout.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(p.tensors(), want):
            if a is p.pout:
                a, b = a[:sum(LENS)], b[:sum(LENS)]
            assert torch.equal(torch.nan_to_num(a.double()), torch.nan_to_num(b.double()))
        p.dec.logprobs(p.plogits, p.ptok, p.plp, p.ph, p.pids, p.ptop)
        torch.cuda.synchronize()
    assert p.dec.device_status() == 0
    p.dec.close()
