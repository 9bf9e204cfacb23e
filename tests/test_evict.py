"""mcpu_evict_kv against a plain model of its slots: K, V and weights move, so everything is equal bit for bit."""
import numpy as np
import pytest
import torch

gpu = pytest.mark.gpu


def kept_slots(w, n, budget, first, last):
    """The slot that each of the `budget` new slots is filled from."""
    inner = budget - last
    v = np.where(np.isnan(w[first:n - last]), -np.inf, w[first:n - last]).astype(np.float64)
    low = np.isnan(w[first:n - last])  # below -inf
    rank = np.lexsort((np.arange(len(v)), -v, low)) + first
    kept = np.sort(rank[: inner - first])
    src = np.arange(budget)
    holes = np.setdiff1d(np.arange(first, inner), kept)
    src[holes] = kept[kept >= inner]
    src[inner:] = np.arange(n - last, n)
    return src


class Cache:
    def __init__(self, total, hkv, layers, seed, slots=None, weights="normal"):
        rng = np.random.default_rng(seed)
        self.total, self.hkv, self.layers = np.asarray(total), hkv, layers
        B = len(total)
        last = -(-self.total // 16)
        self.width = max(1, int(last.max()))
        self.slots = slots or self.width * 16
        P = int(last.sum()) + 3
        ids = rng.permutation(P)
        self.bt = np.full((B, self.width), -1, np.int32)
        at = 0
        for r in range(B):
            self.bt[r, : last[r]] = ids[at : at + last[r]]
            at += last[r]
        self.pools = torch.from_numpy(rng.integers(-32768, 32767, (2 * layers, P, hkv, 16, 64)).astype(np.int16))
        shape = (layers, B, hkv, self.slots)
        w = rng.standard_normal(shape).astype(np.float32)
        if weights == "ties":
            w = rng.integers(0, 4, shape).astype(np.float32)
        elif weights == "equal":
            w[:] = 0.25
        elif weights == "odd":
            pick = rng.integers(0, 8, shape)
            w = np.select([pick == 0, pick == 1, pick == 2, pick == 3, pick == 4],
                          [np.nan, -np.inf, np.inf, -0.0, 0.0], w).astype(np.float32)
        elif weights == "rising":
            w = np.broadcast_to(np.arange(self.slots, dtype=np.float32), shape).copy()
        elif weights == "falling":
            w = -np.broadcast_to(np.arange(self.slots, dtype=np.float32), shape).copy()
        self.w = w
        self.refs = None

    def run(self, limit, budget, first, last, apart=False, stream=None):
        """(pools, weights, lengths, status bits)"""
        from paper_2608_22167_gb300 import mcpu

        pools = self.pools.cuda().view(torch.bfloat16)
        w = torch.from_numpy(self.w).cuda()
        new = torch.full_like(w, 77.0) if apart else w
        lens = torch.full((len(self.total),), -5, dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        refs = None if self.refs is None else torch.from_numpy(self.refs).cuda()
        torch.cuda.synchronize()
        mcpu.mcpu_evict_kv(mcpu.PoolList(list(pools)), w, torch.from_numpy(self.bt).cuda(),
                           torch.from_numpy(self.total.astype(np.int32)).cuda(), limit, budget, first, last, new, lens,
                           status, page_refs=refs, stream=stream)
        torch.cuda.synchronize()
        return pools.view(torch.int16).cpu(), new.cpu().numpy(), lens.tolist(), int(status)

    def check(self, limit, budget, first, last, apart=False, left=(), status=0, stream=None):
        """Rows in `left` are expected to be left as they are."""
        pools, w, lens, bits = self.run(limit, budget, first, last, apart, stream)
        assert bits == status
        assert lens == [n if n <= limit or r in left else budget for r, n in enumerate(self.total.tolist())]
        got_row = lambda p, r, n, h: p[self.bt[r, np.arange(n) // 16], h, np.arange(n) % 16]  # noqa: E731
        touched = torch.zeros(self.pools.shape[:4], dtype=torch.bool)
        for r, n in enumerate(lens):
            for m in range(self.layers):
                for h in range(self.hkv):
                    src = kept_slots(self.w[m, r, h], int(self.total[r]), budget, first, last) if n < self.total[r] else np.arange(n)
                    assert np.array_equal(w[m, r, h, :n], self.w[m, r, h, src], equal_nan=True), (r, m, h)
                    if apart:
                        assert np.all(w[m, r, h, n:] == 77.0)
                    else:
                        assert np.array_equal(w[m, r, h, self.total[r]:], self.w[m, r, h, self.total[r]:], equal_nan=True)
                    for i in (m, m + self.layers):
                        want = self.pools[i][self.bt[r, src // 16], h, src % 16]
                        assert torch.equal(got_row(pools[i], r, n, h), want), (r, m, h)
                        touched[i][self.bt[r, np.arange(n) // 16], h, np.arange(n) % 16] = True
        same = (pools == self.pools).all(-1)
        assert torch.all(same | touched)  # nothing but the rows' new slots is written


SHAPES = [  # limit, budget, first, last
    (100, 100, 4, 16), (100, 64, 0, 0), (64, 64, 64, 0), (64, 64, 0, 64), (70, 64, 10, 54), (33, 33, 1, 1), (1, 1, 0, 0),
    (1, 1, 0, 1), (16, 16, 0, 8), (150, 149, 17, 100),
]


@gpu
@pytest.mark.parametrize("weights", ["normal", "ties", "equal", "odd", "rising", "falling"])
@pytest.mark.parametrize("apart", [False, True])
def test_slots_that_stay(weights, apart):
    for k, (limit, budget, first, last) in enumerate(SHAPES):
        c = Cache([0, 1, 17, limit, limit + 1, limit + 2, 2 * limit + 30, 400], 2, 2, seed=k, weights=weights)
        c.check(limit, budget, first, last, apart)


@gpu
@pytest.mark.parametrize("weights", ["normal", "ties", "odd"])
def test_long_rows(weights):
    Cache([9000, 2049, 70000, 2048, 4500], 2, 1, seed=3, weights=weights).check(2048, 2048, 4, 700)
    Cache([30000], 1, 1, seed=4, weights=weights).check(20000, 17001, 100, 3)
    Cache([30000, 25001], 1, 1, seed=5, weights=weights).check(25000, 25000, 0, 24000, apart=True)


@gpu
@pytest.mark.parametrize("hkv,layers,rows", [(8, 1, 1), (1, 64, 3), (8, 3, 40), (4, 2, 300)])
def test_batches(hkv, layers, rows):
    rng = np.random.default_rng(rows)
    Cache(rng.integers(0, 300, rows), hkv, layers, seed=rows).check(128, 96, 3, 20)


@gpu
def test_rows_that_share_pages_are_left():
    c = Cache([200, 200, 200, 90], 2, 1, seed=6)
    c.refs = np.zeros(c.pools.shape[1], np.int32)
    c.refs[c.bt[0, 2]] = 1    # holds a key that may be overwritten
    c.refs[c.bt[1, 0]] = 2    # all of it among the first
    c.refs[c.bt[2, 10]] = 1   # past the budget: only read
    c.check(100, 100, 16, 20, left=(0,), status=32)


@gpu
def test_bad_pages_and_lengths():
    c = Cache([200, 200, 210, 90], 2, 1, seed=7)
    c.bt[0, 12] = -1
    c.bt[1, 3] = 10 ** 6
    pools, w, lens, bits = c.run(100, 100, 0, 20)
    assert bits == 1 and lens == [200, 200, 100, 90]
    for r in (0, 1):
        assert np.array_equal(w[:, r], c.w[:, r], equal_nan=True)
    c = Cache([200, 200, 210, 90], 2, 1, seed=7, slots=205)
    pools, w, lens, bits = c.run(100, 100, 0, 20)
    assert bits == 2 and lens == [100, 100, 210, 90] and np.array_equal(w[:, 2], c.w[:, 2])
    c = Cache([200, 200], 2, 1, seed=7)
    c.total = np.array([-3, 300])
    pools, w, lens, bits = c.run(100, 100, 0, 20)
    assert bits == 2 and lens == [-3, 300] and torch.equal(pools, c.pools)


@gpu
def test_missing_pages_before_the_first_slots_do_not_matter():
    c = Cache([200], 2, 1, seed=8)
    c.bt[0, 0] = -1
    pools, w, lens, bits = c.run(100, 100, 16, 20)
    assert bits == 0 and lens == [100]


@gpu
def test_other_streams_and_graphs():
    from paper_2608_22167_gb300 import mcpu

    c = Cache([300, 170, 90], 2, 2, seed=9)
    side = torch.cuda.Stream()
    c.check(128, 100, 4, 30, stream=side)
    pools, w = c.pools.cuda().view(torch.bfloat16), torch.from_numpy(c.w).cuda()
    new, lens = torch.empty_like(w), torch.empty(3, dtype=torch.int32, device="cuda")
    status, bt = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.from_numpy(c.bt).cuda()
    sl, pl = torch.from_numpy(c.total.astype(np.int32)).cuda(), mcpu.PoolList(list(pools))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mcpu.mcpu_evict_kv(pl, w, bt, sl, 128, 100, 4, 30, new, lens, status)
    d = Cache([300, 170, 90], 2, 2, seed=10)
    for total in ([300, 170, 90], [101, 140, 96]):
        d.total = np.array(total)
        pools.view(torch.int16).copy_(d.pools), w.copy_(torch.from_numpy(d.w)), bt.copy_(torch.from_numpy(d.bt))
        sl.copy_(torch.tensor(total, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = d.run(128, 100, 4, 30, apart=True)
        assert lens.tolist() == want[2] and torch.equal(pools.view(torch.int16).cpu(), want[0])
        for r, n in enumerate(want[2]):
            assert np.array_equal(new[:, r, :, :n].cpu().numpy(), want[1][:, r, :, :n])


@gpu
def test_offsets_past_32_bits():
    from paper_2608_22167_gb300 import mcpu

    c = Cache([80, 100], 2, 1, seed=11)
    pages, slots = 2 ** 32 // 4096 + 50, 600_000_000
    pools = torch.empty(2, pages, 2, 16, 64, dtype=torch.int16, device="cuda")
    shift = pages - c.pools.shape[1]
    pools[:, shift:] = c.pools.cuda()
    w = torch.empty(1, 2, 2, slots, device="cuda")
    w[..., : c.slots] = torch.from_numpy(c.w).cuda()
    bt = torch.from_numpy(np.where(c.bt >= 0, c.bt + shift, -1).astype(np.int32)).cuda()
    lens, status = torch.empty(2, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    mcpu.mcpu_evict_kv(mcpu.PoolList(list(pools.view(torch.bfloat16))), w, bt, torch.tensor([80, 100], dtype=torch.int32, device="cuda"),
                       64, 64, 4, 16, w, lens, status)
    want = c.run(64, 64, 4, 16)
    assert int(status) == 0 and lens.tolist() == want[2]
    assert torch.equal(pools[:, shift:].cpu(), want[0])
    assert np.array_equal(w[..., :64].cpu().numpy(), want[1][..., :64])


def _args():
    from paper_2608_22167_gb300 import mcpu

    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t)  # noqa: E731
    pools = mcpu.PoolList([z(5, 2, 16, 64, t=torch.bfloat16) for _ in range(4)])
    return dict(pools=pools, key_weights=z(2, 3, 2, 96, t=torch.float32), block_table=z(3, 6), seq_lens=z(3), limit=64,
                budget=64, keep_first=4, keep_last=16, new_key_weights=z(2, 3, 2, 96, t=torch.float32),
                new_seq_lens=z(3), status_word=z(1), page_refs=z(5), stream=None)


def test_binding_refuses_what_it_would_misread():
    from paper_2608_22167_gb300 import mcpu

    args = _args()
    with pytest.raises(ValueError, match="CUDA device"):  # the arguments as they are get as far as this
        mcpu.mcpu_evict_kv(**args)
    for key, x in args.items():
        if not torch.is_tensor(x):
            continue
        wrong = [x.double() if x.is_floating_point() else x.long()]
        if x.shape[-1] > 1:
            wrong.append(torch.stack([x, x], -1)[..., 0])
        if key not in ("status_word", "seq_lens"):
            wrong.append(x[:-1])
        for bad in wrong:
            with pytest.raises(ValueError, match="^(?!.*CUDA device)"):
                mcpu.mcpu_evict_kv(**dict(args, **{key: bad}))
    big = torch.zeros(2 * 3 * 2 * 96 + 96)
    odd = mcpu.PoolList(args["pools"].pools[:3])
    fp8 = mcpu.PoolList([torch.zeros(5, 2, 2176, dtype=torch.uint8)] * 4)
    for bad in (dict(pools=odd), dict(pools=fp8),
                dict(key_weights=big[:-96].view(2, 3, 2, 96), new_key_weights=big[96:].view(2, 3, 2, 96))):
        with pytest.raises(ValueError, match="^(?!.*CUDA device)"):
            mcpu.mcpu_evict_kv(**dict(args, **bad))


def test_host_checks():
    import ctypes

    from paper_2608_22167_gb300 import mcpu

    P, f = 1 << 20, mcpu._lib.mcpu_evict_kv
    dims = mcpu._pack_dims(3, 0, 6, 5, 2, 2, 64, 16)
    pools = (ctypes.c_void_p * 4)(P, P, P, P)
    ok = [pools, 2, P, 96, P, P, 64, 64, 4, 16, P, dims, P, P + 64, P, None]
    assert f(*[mcpu._pack_dims(0, 0, 6, 5, 2, 2, 64, 16) if i == 11 else x for i, x in enumerate(ok)]) == 0
    for i, bad in ((0, None), (0, (ctypes.c_void_p * 4)(P, P, P, None)), (0, (ctypes.c_void_p * 4)(P, P + 8, P, P)),
                   (1, -1), (1, 65), (2, None), (3, 0), (4, None), (5, None), (6, 63), (7, 0), (7, 19), (8, -1), (9, -1),
                   (8, 49), (10, P + 2), (11, None), (12, None), (13, None), (13, P), (14, None)):
        assert f(*[bad if k == i else x for k, x in enumerate(ok)]) == 1, (i, bad)
    assert f(*[mcpu._pack_dims(3, 0, 6, 5, 2, 2, 64, 32) if k == 11 else x for k, x in enumerate(ok)]) == 2
    if not torch.cuda.is_available():
        assert f(*ok) == 4
