"""Forking, shrinking and copying pages, and compacting accepted paths,
against plain models of the tables, counts and stack (exact)."""
import ctypes

import numpy as np
import pytest
import torch

gpu = pytest.mark.gpu


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()


class Model:
    """Block tables, holder counts and the page stack on the host."""

    def __init__(self, rows, width, pages, seed):
        self.rng = np.random.default_rng(seed)
        self.bt = np.full((rows, width), -1, np.int64)
        self.sl = np.zeros(rows, np.int64)
        self.refs = np.zeros(pages, np.int64)
        self.free = [int(p) for p in self.rng.permutation(pages)]
        self.pages = pages

    def fill(self, r, n, first=0):
        for j in range(first, (n + 15) // 16):
            self.bt[r, j] = self.free.pop()
        self.sl[r] = n

    def fork(self, src, dst):
        cs, cd, exhausted = [], [], False
        for s, d in zip(src, dst):
            n = int(self.sl[s])
            full = n // 16
            self.bt[d] = -1
            self.bt[d, :full] = self.bt[s, :full]
            for p in self.bt[d, :full]:
                if p >= 0:
                    self.refs[p] += 1
            self.sl[d] = n
            cs.append(-1)
            cd.append(-1)
            if n % 16:
                if self.free:
                    self.bt[d, full] = cd[-1] = self.free.pop()
                    cs[-1] = int(self.bt[s, full])
                else:
                    exhausted = True
        return cs, cd, exhausted

    def shrink(self, keep, window=0):
        gone = []
        for r in range(len(self.sl)):
            end = (keep[r] + 15) // 16
            begin = max(0, keep[r] - window + 1) // 16 if window > 0 else 0
            for j in range(self.bt.shape[1]):
                p = int(self.bt[r, j])
                if p >= 0 and not begin <= j < end:
                    self.bt[r, j] = -1
                    self.refs[p] -= 1
                    if self.refs[p] < 0:
                        self.refs[p] = 0
                        gone.append(p)
        self.free += sorted(gone)

    def device(self):
        free = np.zeros(self.pages, np.int64)
        free[:len(self.free)] = self.free
        return dict(bt=_i32(self.bt), sl=_i32(self.sl), refs=_i32(self.refs), free=_i32(free),
                    count=_i32([len(self.free)]), scratch=torch.zeros(64, dtype=torch.int32, device="cuda"),
                    status=torch.zeros(1, dtype=torch.int32, device="cuda"))

    def same(self, d, status=0):
        assert np.array_equal(d["bt"].cpu().numpy(), self.bt)
        assert np.array_equal(d["sl"].cpu().numpy(), self.sl)
        assert np.array_equal(d["refs"].cpu().numpy(), self.refs)
        n = int(d["count"].item())
        assert n == len(self.free) and d["free"][:n].cpu().tolist() == self.free
        assert int(d["status"].item()) == status and not d["scratch"].any()


def _fork(d, src, dst):
    from paper_2608_22167_gb300 import mcpu

    cs, cd = (torch.full((len(src),), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    mcpu.mcpu_fork_block_tables(d["bt"], d["sl"], _i32(src), _i32(dst), d["refs"], d["free"], d["count"], cs, cd,
                                d["scratch"], d["status"])
    return cs, cd


def _shrink(d, keep, window=0):
    from paper_2608_22167_gb300 import mcpu

    mcpu.mcpu_shrink_block_tables(d["bt"], _i32(keep), window, d["refs"], d["free"], d["count"], d["scratch"],
                                  d["status"])


@gpu
@pytest.mark.parametrize("rows,width,pages", [(9, 5, 60), (300, 40, 9001), (2048, 7, 30000)])
def test_rounds_of_forks_and_releases(rows, width, pages):
    m = Model(rows, width, pages, rows)
    g = max(1, rows // 5)
    for r in range(g):
        m.fill(r, int(m.rng.integers(0, width * 16 + 1)))
    d = m.device()
    for _ in range(4):
        n = int(m.rng.integers(1, rows - g + 1))
        src = m.rng.integers(0, g, n)
        dst = g + m.rng.permutation(rows - g)[:n]
        cs, cd = _fork(d, src, dst)
        ms, md, exhausted = m.fork(src, dst)
        assert not exhausted and cs.cpu().tolist() == ms and cd.cpu().tolist() == md
        m.same(d)
        # some samples shrink a little, the rest leave
        keep = m.sl.copy()
        for r in range(g, rows):
            keep[r] = 0 if m.rng.random() < 0.6 else int(m.rng.integers(0, m.sl[r] + 1))
        _shrink(d, keep)
        m.shrink(keep)
        m.same(d)
        keep[g:] = 0  # all samples leave before the next round
        m.sl[g:] = 0
        _shrink(d, keep)
        m.shrink(keep)
        d["sl"].copy_(_i32(m.sl))
        m.same(d)
    # a prompt leaves while a sample still holds its pages, then the sample
    m.fork([0], [g])
    _fork(d, [0], [g])
    for gone in (0, g):
        keep = m.sl.copy()
        keep[gone] = m.sl[gone] = 0
        d["sl"].copy_(_i32(m.sl))
        _shrink(d, keep)
        m.shrink(keep)
        m.same(d)


@gpu
def test_shrink_before_a_window():
    m = Model(40, 64, 3000, 5)
    for r in range(40):
        m.fill(r, int(m.rng.integers(0, 1025)))
    d = m.device()
    for window in (2000, 128, 100, 17, 16, 1):  # each keeps less than the one before
        _shrink(d, m.sl, window)
        m.shrink(m.sl, window)
        m.same(d)


@gpu
def test_fork_with_an_empty_stack():
    from paper_2608_22167_gb300 import mcpu

    m = Model(6, 8, 12, 7)
    m.fill(0, 100)
    m.fill(1, 64)
    m.free = m.free[:1]
    d = m.device()
    cs, cd = _fork(d, [0, 1, 0, 0], [2, 3, 4, 5])
    ms, md, exhausted = m.fork([0, 1, 0, 0], [2, 3, 4, 5])
    assert exhausted and cs.cpu().tolist() == ms and cd.cpu().tolist() == md
    m.same(d, mcpu.STATUS_POOL_EXHAUSTED)


@gpu
def test_invalid_rows_pages_and_double_releases():
    from paper_2608_22167_gb300 import mcpu

    m = Model(6, 8, 60, 8)
    m.fill(0, 100)
    m.fill(1, 40)
    d = m.device()
    cs, cd = _fork(d, [0, 9, 0, -1, 1], [2, 3, 0, 4, 77])  # only the first is a valid pair
    ms, md, _ = m.fork([0], [2])
    assert cs.cpu().tolist() == ms + [-1] * 4 and cd.cpu().tolist() == md + [-1] * 4
    m.same(d, mcpu.STATUS_BAD_LENGTHS)
    d["status"].zero_()
    # lengths outside the table: the row is left alone
    keep = m.sl.copy()
    keep[0], keep[1] = -1, 129
    _shrink(d, keep)
    m.same(d, mcpu.STATUS_BAD_LENGTHS)
    d["status"].zero_()
    # an entry outside the pool is cleared and reported
    d["bt"][5, 3] = 60
    _shrink(d, m.sl)
    m.same(d, mcpu.STATUS_BAD_PAGE)
    d["status"].zero_()
    # a page in two tables without a holder count: it returns once
    d["bt"][5, 0] = int(m.bt[1, 0])
    keep = m.sl.copy()
    keep[1] = 0
    m.sl[1] = 0
    d["sl"][1] = 0
    _shrink(d, keep)
    m.shrink(keep)
    m.same(d, mcpu.STATUS_BAD_PAGE)


@gpu
@pytest.mark.parametrize("shape,dtype", [((50, 8, 16, 64), torch.bfloat16), ((50, 1, 16, 64), torch.bfloat16),
                                         ((50, 3, 2176), torch.uint8)])
@pytest.mark.parametrize("pools", [1, 3, 128])
def test_copy_pages(shape, dtype, pools):
    from paper_2608_22167_gb300 import mcpu

    rng = np.random.default_rng(pools)
    raw = [torch.from_numpy(rng.integers(0, 256, (shape[0], int(np.prod(shape[1:])) * dtype.itemsize), dtype=np.uint8))
           for _ in range(pools)]
    dev = [r.cuda().view(dtype).view(shape) for r in raw]
    perm = rng.permutation(50)
    src = np.concatenate([perm[:5], perm[:5], [-1, 4]])
    dst = np.concatenate([perm[5:15], [3, -1]])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mcpu.mcpu_copy_pages(mcpu.PoolList(dev), _i32(src), _i32(dst), status)
    for r, x in zip(raw, dev):
        want = r.clone()
        want[perm[5:15]] = r[src[:10]]
        assert torch.equal(x.view(torch.uint8).view(50, -1).cpu(), want)
    assert int(status.item()) == 0
    mcpu.mcpu_copy_pages(mcpu.PoolList(dev), _i32([50, 1]), _i32([1, 50]), status)
    assert int(status.item()) == mcpu.STATUS_BAD_PAGE


def _compact_case(ctx, lens, taken, hkv, pools, seed, most=None):
    rng = np.random.default_rng(seed)
    ctx, lens, taken = (np.asarray(x, np.int64) for x in (ctx, lens, taken))
    S = ctx + lens
    last = (S + 15) // 16
    P = int(last.sum()) + 1
    ids = rng.permutation(P)
    bt = np.full((len(S), max(1, int(last.max()))), -1, np.int64)
    k = 0
    for r in range(len(S)):
        bt[r, :last[r]] = ids[k:k + last[r]]
        k += int(last[r])
    most = most or max(1, int(taken.max()))
    path = np.full((len(S), most), 12345, np.int64)
    for r in range(len(S)):
        path[r, :taken[r]] = np.sort(rng.permutation(int(lens[r]))[:taken[r]])
    host = [torch.from_numpy(rng.integers(-30000, 30000, (P, hkv, 16, 64)).astype(np.int16)) for _ in range(pools)]
    return dict(ctx=ctx, lens=lens, taken=taken, S=S, bt=bt, path=path, host=host,
                dev=[h.cuda().view(torch.bfloat16) for h in host], new=_i32(np.full(len(S), -5)),
                status=torch.zeros(1, dtype=torch.int32, device="cuda"))


def _compact(c):
    from paper_2608_22167_gb300 import mcpu

    qsl = np.concatenate([[0], np.cumsum(c["lens"])])
    mcpu.mcpu_compact_kv(mcpu.PoolList(c["dev"]), _i32(c["bt"]), _i32(c["S"]), _i32(qsl), _i32(c["path"]),
                         _i32(c["taken"]), c["new"], c["status"])


def _compact_same(c, skip=()):
    for h, x in zip(c["host"], c["dev"]):
        want = h.clone()
        for r in range(len(c["S"])):
            if r in skip:
                continue
            old = c["ctx"][r] + c["path"][r, :c["taken"][r]]
            new = c["ctx"][r] + np.arange(c["taken"][r])
            want[c["bt"][r, new // 16], :, new % 16] = h[c["bt"][r, old // 16], :, old % 16]
        assert torch.equal(x.view(torch.int16).cpu(), want)
    want = [int(c["S"][r]) if r in skip else int(c["ctx"][r] + c["taken"][r]) for r in range(len(c["S"]))]
    assert c["new"].cpu().tolist() == want


@gpu
@pytest.mark.parametrize("hkv,pools", [(8, 2), (2, 1), (1, 5), (3, 128), (16, 7)])
def test_compact(hkv, pools):
    rng = np.random.default_rng(hkv)
    ctx = np.concatenate([[0, 15, 16, 1, 255], rng.integers(0, 100, 20)])
    lens = np.concatenate([[1, 2, 0, 300, 33], rng.integers(0, 64, 20)])
    taken = np.array([int(rng.integers(0, n + 1)) for n in lens])
    taken[3] = 290
    c = _compact_case(ctx, lens, taken, hkv, pools, 3)
    _compact(c)
    _compact_same(c)
    assert int(c["status"].item()) == 0


@gpu
def test_compact_leaves_wrong_rows_alone():
    from paper_2608_22167_gb300 import mcpu

    c = _compact_case([5, 6, 7, 8, 9, 10, 40], [9] * 7, [4, 4, 4, 4, 4, 4, 4], 2, 3, 4, most=6)
    c["path"][0, :4] = [1, 1, 2, 3]    # not increasing
    c["path"][1, :4] = [0, 2, 4, 9]    # past the nodes
    c["path"][2, :4] = [-1, 0, 1, 2]
    c["taken"][3] = 7                  # more than the path holds
    c["taken"][4] = -1
    _compact(c)
    _compact_same(c, skip=(0, 1, 2, 3, 4))
    assert int(c["status"].item()) == mcpu.STATUS_BAD_LENGTHS
    c = _compact_case([5, 30], [20, 9], [3, 4], 2, 3, 5)
    c["path"][0] = [1, 3, 15, 0][:c["path"].shape[1]]
    good = c["bt"].copy()
    c["bt"][0, 1] = 1 << 20
    _compact(c)
    c["bt"] = good
    _compact_same(c, skip=(0,))
    assert int(c["status"].item()) == mcpu.STATUS_BAD_PAGE


def test_host_checks():
    from paper_2608_22167_gb300 import mcpu

    P = 1 << 20
    D = mcpu.Dims
    lib = mcpu._lib
    ptrs = (ctypes.c_void_p * 3)(P, P, P)
    odd = (ctypes.c_void_p * 3)(P, P + 8, P)
    nul = (ctypes.c_void_p * 3)(P, None, P)
    d, d0 = D(4, 9, 19, 34, 2, 2, 64, 16), D(0, 0, 19, 34, 2, 2, 64, 16)
    bad = D(4, 9, 19, -1, 2, 2, 64, 16)

    def compact(pools=ptrs, n=3, bt=P, sl=P, qsl=P, path=P, most=4, taken=P, dims=d, new=P + 64, st=P):
        return lib.mcpu_compact_kv(pools, n, bt, sl, qsl, path, most, taken, ctypes.byref(dims), new, st, None)

    assert compact(pools=None) == 1 and compact(pools=odd) == 1 and compact(pools=nul) == 1
    assert compact(n=-1) == 1 and compact(n=129) == 1 and compact(most=-1) == 1 and compact(path=None) == 1
    assert compact(new=P) == 1 and compact(st=None) == 1 and compact(taken=P + 2) == 1 and compact(bt=None) == 1
    assert compact(dims=bad) == 1 and compact(dims=D(4, 9, 19, 34, 2, 2, 32, 16)) == 2 and compact(dims=d0) == 0

    def fork(n=3, dims=d, **kw):
        names = ("bt", "sl", "src", "dst", "refs", "free", "count", "cs", "cd", "scratch", "st")
        a = [kw.get(k, P) for k in names]
        return lib.mcpu_fork_block_tables(*a[:4], n, ctypes.byref(dims), *a[4:], None)

    for k in ("bt", "sl", "src", "dst", "refs", "free", "count", "cs", "cd", "scratch", "st"):
        assert fork(**{k: None}) == 1 and fork(**{k: P + 1}) == 1, k
    assert fork(n=-1) == 1 and fork(n=2049) == 2 and fork(n=0) == 0 and fork(dims=bad) == 1

    def shrink(dims=d, **kw):
        a = [kw.get(k, P) for k in ("bt", "sl", "refs", "free", "count", "scratch", "st")]
        return lib.mcpu_shrink_block_tables(*a[:2], 0, ctypes.byref(dims), *a[2:], None)

    for k in ("bt", "sl", "refs", "free", "count", "scratch", "st"):
        assert shrink(**{k: None}) == 1 and shrink(**{k: P + 1}) == 1, k
    assert shrink(dims=bad) == 1 and shrink(dims=d0) == 0

    def copy(pools=ptrs, n=3, size=2048, pages=9, cs=P, cd=P, m=4, st=P):
        return lib.mcpu_copy_pages(pools, n, size, pages, cs, cd, m, st, None)

    assert copy(pools=odd) == 1 and copy(size=0) == 1 and copy(size=24) == 1 and copy(pages=-1) == 1 and copy(m=-1) == 1
    assert copy(cs=None) == 1 and copy(cd=P + 2) == 1 and copy(st=None) == 1 and copy(m=0) == 0 and copy(n=0) == 0
    assert copy(size=1 << 31) == 2


def test_pool_lists():
    from paper_2608_22167_gb300 import mcpu

    a, b = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    assert mcpu.PoolList([a, a.clone()]).page_bytes == 2 * 2048
    for bad in ([], [a, b], [a, a.half()], [a[:, :1]], [a] * 129):
        with pytest.raises(ValueError):
            mcpu.PoolList(bad)
    with pytest.raises(ValueError):
        mcpu.mcpu_compact_kv(mcpu.PoolList([torch.zeros(3, 2, 2176, dtype=torch.uint8)]), None, None, None, None, None,
                             None, None)


def _grow_from(d, seq_lens, context_lens):
    from paper_2608_22167_gb300 import mcpu

    mcpu.mcpu_grow_block_tables_from(d["bt"], _i32(seq_lens), _i32(context_lens), d["free"], d["count"], d["status"])


def _grown(m, d, new):
    """Checks the tables after growing the model's rows to `new` lengths, and takes over which page went where."""
    n = int(d["count"].item())
    popped, m.free = m.free[n:], m.free[:n]
    bt = d["bt"].cpu().numpy()
    got = []
    for r in range(len(new)):
        first, end = -(-int(m.sl[r]) // 16), max(-(-int(new[r]) // 16), -(-int(m.sl[r]) // 16))
        assert np.array_equal(bt[r, :first], m.bt[r, :first]) and np.all(bt[r, end:] == -1)
        got += [int(p) for old, p in zip(m.bt[r, first:end], bt[r, first:end]) if old < 0]
        m.bt[r, first:end] = bt[r, first:end]
    assert sorted(got) == sorted(popped) and min(got, default=0) >= 0
    m.sl = np.asarray(new).copy()


@gpu
@pytest.mark.parametrize("window", [1, 16, 50, 128])
def test_growing_keeps_what_a_window_released(window):
    # rows of up to 600 tokens whose windows need 40 x (9 + 4) pages at most: a pool without room for their tables
    m = Model(40, 64, 40 * 13, window)
    for r in range(40):
        m.fill(r, int(m.rng.integers(0, 130)))
    d = m.device()
    for _ in range(10):
        _shrink(d, m.sl, window)
        m.shrink(m.sl, window)
        d["sl"].copy_(_i32(m.sl))
        m.same(d)
        new = m.sl + m.rng.integers(0, 49, 40) * (m.rng.random(40) < 0.8)
        _grow_from(d, new, m.sl)
        _grown(m, d, new)
        d["sl"].copy_(_i32(m.sl))
        m.same(d)
    # forked rows keep the missing entries of their source
    m.sl[30:] = 0
    _shrink(d, m.sl, window)
    m.shrink(m.sl, window)
    d["sl"].copy_(_i32(m.sl))
    _fork(d, range(10), range(30, 40))
    m.fork(range(10), range(30, 40))
    m.same(d)
    new = m.sl + 20
    _grow_from(d, new, m.sl)
    _grown(m, d, new)
    assert int(d["status"].item()) == 0


@gpu
def test_growing_does_not_replace_a_missing_page_of_the_context():
    from paper_2608_22167_gb300 import mcpu

    m = Model(3, 8, 30, 9)
    m.fill(0, 60)
    m.free, left = [], m.free
    d = m.device()
    _fork(d, [0], [1])  # no page for the partial last one
    m.fork([0], [1])
    m.same(d, mcpu.STATUS_POOL_EXHAUSTED)
    d["status"].zero_()
    m.free = left
    d = m.device()
    new = np.array([60, 70, 5])
    _grow_from(d, new, m.sl)
    _grown(m, d, new)
    assert m.bt[1, 3] == -1 and int(d["status"].item()) == 0
    # lengths that grow by nothing, a context longer than the row, and a negative one
    _grow_from(d, [60, 20, 0], [60, 70, 0])
    assert np.array_equal(d["bt"].cpu().numpy(), m.bt) and int(d["status"].item()) == 0
    _grow_from(d, [60, 20, 20], [60, 70, -1])
    assert np.array_equal(d["bt"].cpu().numpy(), m.bt) and int(d["status"].item()) == mcpu.STATUS_BAD_LENGTHS


def test_grow_from_host_checks():
    from paper_2608_22167_gb300 import mcpu

    P = 1 << 20
    ok = dict(bt=P, sl=P, ctx=P, dims=mcpu.Dims(4, 0, 19, 0, 1, 1, 64, 16), refs=None, free=P, count=P, cs=None, cd=None,
              st=P)

    def call(**kw):
        a = dict(ok, **kw)
        return mcpu._lib.mcpu_grow_block_tables_from(a["bt"], a["sl"], a["ctx"], a["dims"] and ctypes.byref(a["dims"]),
                                                     a["refs"], a["free"], a["count"], a["cs"], a["cd"], a["st"], None)

    for name in ("bt", "sl", "ctx", "free", "count", "st"):
        assert call(**{name: None}) == 1 and call(**{name: P + 2}) == 1, name
    assert call(dims=None) == 1 and call(dims=mcpu.Dims(-1, 0, 19, 0, 1, 1, 64, 16)) == 1
    assert call(dims=mcpu.Dims(4, 0, 1 << 28, 0, 1, 1, 64, 16)) == 2
    assert call(dims=mcpu.Dims(0, 0, 19, 0, 1, 1, 64, 16)) == 0
    assert call(dims=mcpu.Dims(4, 0, 19, -1, 1, 1, 64, 16)) == 1
    for some in (dict(refs=P), dict(cs=P), dict(cd=P), dict(refs=P, cs=P), dict(refs=P, cd=P), dict(cs=P, cd=P),
                 dict(refs=P + 2, cs=P, cd=P), dict(refs=P, cs=P + 2, cd=P), dict(refs=P, cs=P, cd=P + 2)):
        assert call(**some) == 1, some
    bt, sl = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    good = dict(block_table=bt, seq_lens=sl, context_lens=sl, free_pages=sl, free_count=sl[:1], status_word=sl[:1],
                stream=object())
    for bad in (dict(context_lens=sl[:1]), dict(context_lens=sl.long()), dict(seq_lens=sl.long()),
                dict(block_table=bt[:, :2]), dict(page_refs=sl), dict(page_refs=sl, copy_src=sl, copy_dst=sl[:1]),
                dict(page_refs=sl.long(), copy_src=sl, copy_dst=sl)):
        with pytest.raises(ValueError):
            mcpu.mcpu_grow_block_tables_from(**dict(good, **bad))


@gpu
def test_rows_that_end_inside_a_shared_page_get_their_own():
    # samples shortened into the full pages they share with their prompt, then grown and appended to: the prompt and
    # the other samples keep their K and V, the appending row keeps what it had
    from paper_2608_22167_gb300 import mcpu

    rng = np.random.default_rng(12)
    rows, hkv, pages = 14, 2, 200
    m = Model(rows, 10, pages, 12)
    m.fill(0, 133)
    m.fill(1, 96)
    src, dst = [0, 0, 0, 0, 0, 0, 1, 1, 1, 1, 1, 1], list(range(2, 14))
    m.fork(src, dst)
    d = m.device()
    pools = [torch.from_numpy(rng.standard_normal((pages, hkv, 16, 64)).astype(np.float32)).bfloat16().cuda()
             for _ in range(2)]
    # row 1 itself is shortened into a page its samples hold, three samples to the same one
    keep = np.array([133, 90, 70, 71, 133, 64, 0, 128, 96, 95, 95, 96, 81, 5])
    _shrink(d, keep)
    m.shrink(keep)
    m.sl = keep.copy()
    d["sl"].copy_(_i32(keep))
    m.same(d)

    def held(r, n):
        pos = torch.arange(n, device="cuda")
        page = d["bt"][r].long()[pos // 16]
        return torch.stack([p[page, :, pos % 16] for p in pools])

    before = [held(r, int(keep[r])) for r in range(rows)]
    grow = np.array([0, 3, 20, 1, 5, 16, 0, 0, 4, 2, 2, 0, 30, 12])
    new = keep + grow
    cs, cd = (torch.full((rows,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    old = d["bt"].cpu().numpy()
    refs = d["refs"].cpu().numpy()
    mcpu.mcpu_grow_block_tables_from(d["bt"], _i32(new), _i32(keep), d["free"], d["count"], d["status"],
                                     page_refs=d["refs"], copy_src=cs, copy_dst=cd)
    mcpu.mcpu_copy_pages(mcpu.PoolList(pools), cs, cd, d["status"])
    assert int(d["status"].item()) == 0
    bt = d["bt"].cpu().numpy()
    # nobody else holds a page that a row is going to write, the counts are those of the table, and what was let go
    # was copied
    used, times = np.unique(bt[bt >= 0], return_counts=True)
    counts = np.zeros(pages, int)
    counts[used] = times - 1
    assert np.array_equal(d["refs"].cpu().numpy(), counts)
    moved = 0
    for r in range(rows):
        for j in range(int(keep[r]) // 16, -(-int(new[r]) // 16) if grow[r] else 0):
            assert bt[r, j] >= 0 and counts[bt[r, j]] == 0
        j = int(keep[r]) // 16
        if grow[r] and keep[r] % 16 and bt[r, j] != old[r, j]:
            assert refs[old[r, j]] > 0 and (int(cs[r]), int(cd[r])) == (old[r, j], bt[r, j])
            moved += 1
        else:
            assert (int(cs[r]), int(cd[r])) == (-1, -1)
        assert np.array_equal(bt[r, :j], old[r, :j])
    assert moved == 7  # rows 1, 2, 3, 9, 10, 12 and 13; others hold each of their pages
    left = int(d["count"].item())
    in_use = set(used.tolist())
    assert len(in_use) + left == pages and not in_use & set(d["free"][:left].tolist())
    x = torch.randn(int(grow.sum()), hkv, 64, device="cuda").bfloat16()
    qsl = _i32(np.concatenate([[0], np.cumsum(grow)]))
    mcpu.mcpu_kv_append(x, x, *pools, d["bt"], _i32(new), qsl, d["status"])
    for r in range(rows):
        assert torch.equal(held(r, int(keep[r])), before[r]), r
    assert int(d["status"].item()) == 0


@gpu
def test_a_shared_page_with_an_empty_stack():
    from paper_2608_22167_gb300 import mcpu

    m = Model(3, 4, 10, 2)
    m.fill(0, 48)
    m.fork([0], [1])
    m.shrink([48, 40, 0])
    m.sl[1] = 40
    m.free = []
    d = m.device()
    cs, cd = (torch.full((3,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    shared = int(m.bt[1, 2])
    mcpu.mcpu_grow_block_tables_from(d["bt"], _i32([48, 41, 0]), _i32([48, 40, 0]), d["free"], d["count"], d["status"],
                                     page_refs=d["refs"], copy_src=cs, copy_dst=cd)
    m.bt[1, 2] = -1
    m.refs[shared] -= 1
    m.same(d, mcpu.STATUS_POOL_EXHAUSTED)
    assert cs.tolist() == [-1] * 3 and cd.tolist() == [-1] * 3


@gpu
def test_one_of_the_rows_that_grow_from_a_page_at_once_may_keep_it():
    from paper_2608_22167_gb300 import mcpu

    m = Model(4, 4, 20, 3)
    m.fill(0, 48)
    m.fork([0, 0, 0], [1, 2, 3])
    d = m.device()
    _shrink(d, [0, 40, 41, 40])
    keep = _i32([0, 40, 41, 40])
    cs, cd = (torch.full((4,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    shared = int(m.bt[0, 2])
    mcpu.mcpu_grow_block_tables_from(d["bt"], keep + 2, keep, d["free"], d["count"], d["status"], page_refs=d["refs"],
                                     copy_src=cs, copy_dst=cd)
    tails = d["bt"][1:, 2].tolist()
    assert tails.count(shared) == 1 and len(set(tails)) == 3 and int(d["refs"][shared]) == 0
    assert [int(s) for s in cs[1:]] == [-1 if t == shared else shared for t in tails]
    assert [int(s) for s in cd[1:]] == [-1 if t == shared else t for t in tails]
    # in use: the prompt's three pages, two in place of the shared one, one that row 0's two tokens open
    assert int(cs[0]) == int(cd[0]) == -1 and int(d["status"].item()) == 0 and int(d["count"].item()) == 20 - 6


@gpu
@pytest.mark.parametrize("at", [0, 5, 127, 511, 512, 700])
def test_a_fork_into_a_row_that_holds_a_page_is_reported(at):
    from paper_2608_22167_gb300 import mcpu

    m = Model(4, 701, 900, at)
    m.fill(0, 100)
    d = m.device()
    lost = m.free[0]  # never popped here
    d["bt"][2, at] = lost
    cs, cd = _fork(d, [0, 0], [1, 3])
    ms, md, _ = m.fork([0, 0], [1, 3])
    m.bt[2, at] = lost
    m.same(d)  # the others' forks are fine
    _fork(d, [0], [2])
    m.fork([0], [2])
    m.same(d, mcpu.STATUS_BAD_PAGE)


@pytest.mark.parametrize("pages", [0x7fff0000, 0x7fffffff])
def test_page_counts_that_do_not_fit_are_refused(pages):
    # dividing so many pages into segments would pass 32 bits
    from paper_2608_22167_gb300 import mcpu

    P = 1 << 20
    d = mcpu.Dims(4, 0, 19, pages, 1, 1, 64, 16)
    assert mcpu._lib.mcpu_shrink_block_tables(P, P, 0, ctypes.byref(d), P, P, P, P, P, None) == 2
    assert mcpu._lib.mcpu_fork_block_tables(P, P, P, P, 3, ctypes.byref(d), P, P, P, P, P, P, P, None) == 2
