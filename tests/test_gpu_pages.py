"""ent_cache_fork, ent_cache_release and ent_cache_compact against the oracle: tables,
lengths, share counts, free lists, flags and every block's contents, bit for bit."""
import numpy as np
import pytest

from oracle import pages as OG
from tests.prompt_data import config
from tests.test_gpu_parity import torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu


class Pool:
    """R sequences in a pool of P blocks, on the host and on the GPU."""

    def __init__(self, torch, lens, R, P, maxb, kind="bf16", H=2, D=64, seed=0, pad=0, ksum=True):
        rng = np.random.default_rng(seed)
        self.torch, self.P, self.R, self.maxb, self.kind = torch, P, R, maxb, kind
        self.cfg = config(H, H, D, "f32" if kind == "f32" else "bf16", max_batch=max(R, 1),
                          max_blocks_per_seq=maxb, num_pool_blocks=P, scoring=int(not ksum))
        self.tables = rng.integers(-5, P + 5, (R, maxb))       # what no sequence holds is anything
        self.ctx, self.shared = np.zeros(R, np.int64), np.zeros(P, np.int64)
        ids = rng.permutation(P)
        at = 0
        for b, n in enumerate(lens):
            nb = -(-n // 16)
            self.tables[b, :nb] = ids[at:at + nb]
            self.ctx[b] = n
            at += nb
        self.ids = np.concatenate([ids, np.full(pad, -9)])
        self.free = [at, P]
        shapes = [(P, H, 16, D), (P, H, D, 16)] + ([(P, H, D)] if ksum else []) + [(P, H)] * 2 * (kind == "q8")
        top = {"f32": 1 << 31, "bf16": 1 << 15, "q8": 256}[kind]
        np_t = {"f32": np.int32, "bf16": np.int16, "q8": np.uint8}[kind]
        self.pools = [rng.integers(0, top, s).astype(np_t) if i < 2 else rng.random(s).astype(np.float32)
                      for i, s in enumerate(shapes)]

    def upload(self):
        t = lambda x: self.torch.tensor(np.asarray(x), device="cuda:0")  # noqa: E731
        i32 = lambda x: t(np.asarray(x, np.int32))  # noqa: E731
        self.d = dict(tables=i32(self.tables), ctx=i32(self.ctx), shared=i32(self.shared), ids=i32(self.ids),
                      free=i32(self.free))
        self.dp = [t(x) for x in self.pools]
        self.used = i32([-7])

    def caches(self):
        k, v = self.dp[:2]
        ksum = self.dp[2] if self.cfg["scoring"] == 0 else None
        sc = self.dp[-2:] if self.kind == "q8" else [None, None]
        return k, v, ksum, sc

    def call(self, dec, what, *rows, shared=True, stream=None):
        d = self.d
        k, v, ksum, sc = self.caches()
        i32 = lambda x: self.torch.tensor(np.asarray(x), dtype=self.torch.int32, device="cuda:0")  # noqa: E731
        sh = d["shared"] if shared else None
        rows = [i32(r) for r in rows]
        if stream is not None:
            self.torch.cuda.synchronize()
        if what == "fork":
            dec.fork(*rows, d["tables"], d["ctx"], sh, d["ids"], d["free"], k, v, ksum, *sc, stream=stream)
        elif what == "release":
            dec.release(rows[0], d["tables"], d["ctx"], d["ids"], d["free"], sh, stream=stream)
        else:
            dec.compact(d["tables"], d["ctx"], d["ids"], d["free"], k, v, ksum, sh, *sc, n_used=self.used,
                        stream=stream)
        self.torch.cuda.synchronize()
        return dec.device_status()

    def oracle(self, what, *rows, shared=True):
        sh = self.shared if shared else None
        if what == "fork":
            return OG.fork(*rows, self.tables, self.ctx, sh, self.ids, self.free, self.P, self.pools)
        if what == "release":
            return OG.release(rows[0], self.tables, self.ctx, sh, self.ids, self.free, self.P)
        flags, self.count = OG.compact(self.tables, self.ctx, sh, self.ids, self.free, self.P, self.pools)
        return flags

    def same(self):
        for name in ("tables", "ctx", "shared", "ids", "free"):
            got, ref = self.d[name].cpu().numpy(), np.asarray(getattr(self, name))
            assert np.array_equal(got, ref), (name, np.argwhere(got != ref)[:5])
        for i, (got, ref) in enumerate(zip(self.dp, self.pools)):
            assert np.array_equal(got.cpu().numpy(), ref), (i, np.argwhere((got.cpu().numpy() != ref).reshape(self.P, -1).any(1))[:5])

    def both(self, dec, what, *rows, shared=True, flags=None):
        want = self.oracle(what, *rows, shared=shared)
        got = self.call(dec, what, *rows, shared=shared)
        assert got == want and (flags is None or got == flags), (got, want)
        self.same()
        if what == "compact":
            assert int(self.used[0]) == self.count


def decoder(p):
    from paper_2603_03310_amd.runner import Decoder
    return Decoder(**p.cfg)


KINDS = [("bf16", 2, 64), ("bf16", 8, 128), ("f32", 1, 64), ("f32", 5, 128), ("q8", 1, 64), ("q8", 3, 128)]


@pytest.mark.parametrize("kind,H,D", KINDS)
def test_fork_release_compact(torch_cuda, kind, H, D):
    """Samples and samples of samples; some end; the rest move together; all end."""
    lens = [0, 1, 15, 16, 17, 100, 256, 255, 33]
    p = Pool(torch_cuda, lens, 24, 200, 20, kind, H, D, seed=H)
    p.upload()
    with decoder(p) as dec:
        p.both(dec, "fork", [5, 5, 1, 0, 3, 7], [9, 10, 11, 12, 13, 14], flags=0)
        p.both(dec, "fork", [9, 14, 4], [15, 16, 17], flags=0)
        p.both(dec, "release", [5, 11, 2, 0], flags=0)
        p.both(dec, "release", [7, 14, 16], flags=0)
        p.both(dec, "compact", flags=0)
        p.both(dec, "fork", [9, 10, 8], [5, 7, 14], flags=0)
        p.both(dec, "compact", flags=0)
        p.both(dec, "release", np.arange(24), flags=0)
        assert (p.shared == 0).all() and p.free == [0, 200] and sorted(p.ids) == list(range(200))
        p.both(dec, "compact", flags=0)
        assert p.count == 0


def test_a_full_pool_and_single_blocks(torch_cuda):
    """All blocks in use (also where their number is a whole number of words), and pools of a few."""
    for P in (1, 31, 32, 33, 64, 200):
        p = Pool(torch_cuda, [16 * P], 3, P, max(P, 2), seed=P)
        p.upload()
        with decoder(p) as dec:
            p.both(dec, "compact", flags=0)
            p.both(dec, "fork", [0], [2], flags=0)
            p.both(dec, "release", [0], flags=0)
            p.both(dec, "compact", flags=0)
            p.both(dec, "release", [2], flags=0)
            assert p.free == [0, P]
            p.both(dec, "compact", flags=0)


def test_large(torch_cuda):
    """Thousands of rows and blocks, many holders of a block, sequences of many blocks."""
    rng = np.random.default_rng(5)
    lens = list(rng.integers(0, 700, 300)) + [16 * 3000 + 5]
    P = sum(-(-n // 16) for n in lens) + 2500
    p = Pool(torch_cuda, lens, 2400, P, 3002, "q8", 1, 64, seed=1)
    p.upload()
    with decoder(p) as dec:
        src = np.concatenate([rng.integers(0, 300, 1900), [300] * 99])
        dst = 301 + rng.permutation(2099)[:1999]
        p.both(dec, "fork", src, dst, flags=0)
        p.both(dec, "release", rng.permutation(2400)[:1500], flags=0)
        p.both(dec, "compact", flags=0)
        p.both(dec, "release", rng.permutation(2400), flags=0)
        assert p.free == [0, P] and (p.shared == 0).all()


def test_the_list_runs_out(torch_cuda):
    p = Pool(torch_cuda, [17, 40, 32, 0], 12, 8, 4, seed=2)     # 2 + 3 + 2 blocks: one is free
    p.upload()
    with decoder(p) as dec:
        p.both(dec, "fork", [2, 3, 0, 1, 2], [4, 5, 6, 7, 8], flags=OG.CACHE_FULL)
        assert p.ctx[6] == 17 and p.ctx[7] == p.ctx[8] == 0
        p.both(dec, "fork", [2, 3], [9, 10], flags=0)           # those that need none go on
        p.both(dec, "release", [6, 1], flags=0)
        p.both(dec, "fork", [0], [7], flags=0)


def test_bad_rows_lengths_tables_and_ids(torch_cuda):
    big = (1 << 31) - 1
    p = Pool(torch_cuda, [20, 33, 64, 5, 16, 48, 20], 16, 40, 4, seed=3)
    p.tables[1, 0], p.tables[2, 3], p.tables[5, 1] = 40, -1, big
    p.tables[6, 1] = -3                                         # the block that it is writing
    p.ctx[3], p.ctx[4], p.ctx[15] = -1, 65, big
    p.ids[p.free[0] + 1] = 40
    p.upload()
    with decoder(p) as dec:
        # A row twice, a source as destination, rows outside, lengths outside.
        p.both(dec, "fork", [0, 0, 2, 7, -1, 16, 0, 0, big, 3, 4, 15], [7, 7, 0, 8, 9, 9, 16, -1, 10, 11, 12, 13])
        p.both(dec, "fork", [0, 1, 6, 2, 5], [8, 9, 10, 11, 12])   # the second gets the id outside
        assert -1 in p.tables[9]
        p.both(dec, "compact")
        p.both(dec, "release", [0, 0, 9, -1, 16, big, 3, 15, 10, 11, 5])
        p.both(dec, "release", [0, 9])                             # already over
        p.both(dec, "compact")


def test_blocks_listed_too_often(torch_cuda):
    """A block that sequences hold without a share: freed once; in one call and in two."""
    p = Pool(torch_cuda, [64, 64, 64, 64], 6, 30, 5, seed=4)
    p.tables[1] = p.tables[0]
    p.tables[2, 2] = p.tables[2, 3]
    p.upload()
    with decoder(p) as dec:
        p.both(dec, "release", [0, 1, 2], flags=OG.BAD_TABLE)
        p.both(dec, "release", [3], flags=0)
        p.both(dec, "compact", flags=0)
    p = Pool(torch_cuda, [64, 64], 6, 30, 5, seed=4)
    p.tables[1, 0] = p.tables[0, 3]
    p.upload()
    with decoder(p) as dec:
        p.both(dec, "release", [0, 1], shared=False, flags=OG.BAD_TABLE)
        p.both(dec, "release", [0, 1], shared=False, flags=0)


@pytest.mark.parametrize("free", [[-1, 3], [5, 4], [0, 1 << 30], [41, 41], [-(1 << 31), 0]], ids=str)
def test_bad_free_ranges_change_nothing(torch_cuda, free):
    p = Pool(torch_cuda, [20, 33], 4, 40, 4, seed=5)
    good, p.free = p.free, list(free)
    p.upload()
    with decoder(p) as dec:
        before = [p.tables.copy(), p.ctx.copy(), p.shared.copy()]
        p.both(dec, "fork", [0], [2], flags=OG.BAD_TABLE)
        p.both(dec, "release", [1], flags=OG.BAD_TABLE)
        for a, b in zip(before, (p.tables, p.ctx, p.shared)):
            assert np.array_equal(a, b)
        p.free = list(good)
        p.d["free"].copy_(torch_cuda.tensor(good, dtype=torch_cuda.int32))
        p.both(dec, "fork", [0], [2], flags=0)
        p.both(dec, "release", [1, 0], flags=0)
        p.d["free"].fill_(-5)
        p.both(dec, "compact", flags=0)                          # whatever the range held


def test_no_room_below_the_list(torch_cuda):
    """Blocks that never came from the list: the highest ids that fit."""
    p = Pool(torch_cuda, [100, 60], 3, 40, 8, seed=6, pad=4)
    p.free = [3, 10]
    p.upload()
    with decoder(p) as dec:
        p.both(dec, "release", [1, 0], flags=OG.CACHE_FULL)
        p.both(dec, "compact", flags=0)                          # a list longer than the pool


def test_without_shares_and_summaries(torch_cuda):
    p = Pool(torch_cuda, [100, 60, 16, 3], 6, 60, 8, seed=7, ksum=False)
    p.upload()
    with decoder(p) as dec:
        p.both(dec, "release", [2, 0], shared=False, flags=0)
        p.both(dec, "compact", shared=False, flags=0)
        p.both(dec, "fork", [1, 3], [0, 2], flags=0)


def test_captured_and_replayed(torch_cuda):
    """A fork, a release and a compact in one graph, replayed on the same state: the eager
    result each time, with eager calls of the same context between the replays."""
    torch = torch_cuda
    p = Pool(torch, [100, 60, 16, 3], 8, 60, 8, seed=8)
    p.upload()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    src, dst, end = i32([0, 1, 0]), i32([4, 5, 6]), i32([0, 2, 5])
    with decoder(p) as dec:
        k, v, ksum, sc = p.caches()
        d = p.d

        def work():
            dec.fork(src, dst, d["tables"], d["ctx"], d["shared"], d["ids"], d["free"], k, v, ksum)
            dec.release(end, d["tables"], d["ctx"], d["ids"], d["free"], d["shared"])
            dec.compact(d["tables"], d["ctx"], d["ids"], d["free"], k, v, ksum, d["shared"], n_used=p.used)

        state = list(d.values()) + p.dp + [p.used]
        saved = [t.clone() for t in state]
        s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            work()
        for what, rows in (("fork", ([0, 1, 0], [4, 5, 6])), ("release", ([0, 2, 5],)), ("compact", ())):
            assert p.oracle(what, *rows) == 0
        for _ in range(4):
            for t, x in zip(state, saved):
                t.copy_(x)
            g.replay()
            torch.cuda.synchronize()
            p.same()
            assert int(p.used[0]) == p.count
            dec.release(i32([4]), d["tables"], d["ctx"], d["ids"], d["free"], d["shared"])
            torch.cuda.synchronize()
        assert dec.device_status() == 0


def test_another_stream(torch_cuda):
    torch = torch_cuda
    p = Pool(torch, [100, 60, 16, 3], 8, 60, 8, seed=15)
    p.upload()
    s = torch.cuda.Stream()
    with decoder(p) as dec:
        for what, rows in (("fork", ([0, 1, 0], [4, 5, 6])), ("release", ([0, 2, 5],)), ("compact", ())):
            assert p.oracle(what, *rows) == 0
            s.wait_stream(torch.cuda.current_stream())
            p.call(dec, what, *rows, stream=s)
            p.same()


def test_refusals(torch_cuda):
    torch = torch_cuda
    from paper_2603_03310_amd import ent
    p = Pool(torch, [20, 33], 4, 40, 4, seed=9)
    p.upload()
    d = p.d
    k, v, ksum, _ = p.caches()
    sc = torch.ones((40, 2), device="cuda:0")
    rows = torch.tensor([0, 1], dtype=torch.int32, device="cuda:0")
    dst = torch.tensor([2, 3], dtype=torch.int32, device="cuda:0")
    inval, unsup = ent.ENT_E_INVAL, ent.ENT_E_UNSUPPORTED

    def refused(dec, code, what, **kw):
        a = dict(dict(N=2, R=4, rows=rows, dst=dst, tables=d["tables"], ctx=d["ctx"], shared=d["shared"],
                      ids=d["ids"], n_ids=40, free=d["free"], k=k, v=v, ks=None, vs=None, ksum=ksum), **kw)
        tail = (a["tables"], a["ctx"], a["shared"], a["ids"], a["n_ids"], a["free"])
        caches = (a["k"], a["v"], a["ks"], a["vs"], a["ksum"])
        with pytest.raises(ent.EntError) as e:
            if what == "fork":
                ent.ent_cache_fork(dec.ctx, a["N"], a["R"], a["rows"], a["dst"], *tail, *caches)
            elif what == "release":
                ent.ent_cache_release(dec.ctx, a["N"], a["R"], a["rows"], *tail)
            else:
                ent.ent_cache_compact(dec.ctx, a["R"], *tail, *caches)
        assert e.value.code == code, (what, kw, str(e.value))

    with decoder(p) as dec:
        for what in ("fork", "release", "compact"):
            for kw in (dict(R=-1), dict(R=5), dict(n_ids=-1), dict(tables=None), dict(ctx=None), dict(ids=None),
                       dict(free=None)):
                refused(dec, inval, what, **kw)
        for what in ("fork", "release"):
            for kw in (dict(N=-1), dict(N=3, R=2), dict(rows=None)):
                refused(dec, inval, what, **kw)
        for what in ("fork", "compact"):
            for kw in (dict(k=None), dict(v=None), dict(ksum=None), dict(ks=sc), dict(vs=sc),
                       dict(k=k.data_ptr() + 8), dict(ksum=ksum.data_ptr() + 4)):
                refused(dec, inval, what, **kw)
        refused(dec, inval, "fork", dst=None)
        for what, kw in (("fork", dict(rows=d["ctx"])), ("fork", dict(dst=d["ctx"])), ("fork", dict(shared=d["ctx"])),
                         ("release", dict(rows=d["ctx"])), ("release", dict(shared=d["ctx"])),
                         ("release", dict(rows=d["ids"]))):
            refused(dec, inval, what, **kw)
        refused(dec, inval, "fork", shared=None)
        refused(dec, inval, "compact", n_ids=39)
        ent.ent_cache_fork(dec.ctx, 0, 4, *[None] * 6, 0, *[None] * 6)
        ent.ent_cache_release(dec.ctx, 0, 4, *[None] * 5, 0, None)
        ent.ent_cache_compact(dec.ctx, 0, *[None] * 4, 40, *[None] * 6)
        torch.cuda.synchronize()
        p.same()
    q = Pool(torch, [20], 4, 40, 4, "f32", seed=9)
    with decoder(q) as dec:                                     # 8-bit codes need a bf16 context
        refused(dec, unsup, "fork", ks=sc, vs=sc)
        refused(dec, unsup, "compact", ks=sc, vs=sc)


def test_offsets_past_32_bits(torch_cuda):
    """Blocks that lie more than 4 GB into their cache, forked, compacted and freed."""
    torch = torch_cuda
    P, H, D = 140000, 8, 128                                     # 4.6 GB of keys, as many of values
    p = Pool(torch, [20, 40, 16], 5, 300, 4, "bf16", H, D, seed=10)
    order = np.random.default_rng(11).permutation(300) + P - 300
    p.tables = np.where((p.tables >= 0) & (p.tables < 300), order[p.tables % 300], p.tables)
    p.ids = np.concatenate([np.zeros(P - 300, np.int64), order[p.ids]])
    p.free, p.P = [P - 300 + p.free[0], P], P
    p.shared = np.zeros(P, np.int64)
    p.cfg["num_pool_blocks"] = P
    small = p.pools
    wide = [torch.zeros((P,) + x.shape[1:], dtype=torch.tensor(x[:1]).dtype, device="cuda:0") for x in small]
    for w, x in zip(wide, small):
        w[P - 300:] = torch.tensor(x, device="cuda:0")

    class Blocks:                                                # the host's copy of the few blocks that matter
        def __init__(self, x):
            self.at = {P - 300 + i: x[i].copy() for i in range(300)}

        def __getitem__(self, i):
            return self.at[int(i)]

        def __setitem__(self, i, v):
            self.at[int(i)] = np.array(v)

    hosts = [Blocks(x) for x in small]
    p.pools = []
    p.upload()
    p.pools, p.dp = hosts, wide

    def same():
        for name in ("tables", "ctx", "shared", "ids", "free"):
            assert np.array_equal(p.d[name].cpu().numpy(), np.asarray(getattr(p, name))), name
        for h, w in zip(hosts, wide):
            ids = sorted(h.at)
            got = w[torch.tensor(ids, device="cuda:0")].cpu().numpy()
            assert np.array_equal(got, np.stack([h.at[i] for i in ids]))

    p.same = same
    with decoder(p) as dec:
        p.both(dec, "fork", [0, 1], [3, 4], flags=0)
        p.both(dec, "release", [1], flags=0)
        p.both(dec, "compact", flags=0)
        assert p.count == 7 and max(h for h in hosts[0].at) >= P - 300 and 0 in hosts[0].at
        p.both(dec, "release", [0, 2, 3, 4], flags=0)
