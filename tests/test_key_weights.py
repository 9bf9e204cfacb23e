"""mcpu_accumulate_weights against the formula in 64 bits.

Tolerance: a term exp(x), x = scale q . k - lse, is off relatively by the error
of x: 64 products, exact in fp32, are added in fp32 (64 2^-24 scale sum |q_d k_d|,
about 5 for normal values), x 2^-24 for the scaling and lse 2^-24 for its
rounding to base 2, so below 64 5 2^-24 + 32 2^-24 < 2.2e-5; 2^x itself is good to
2^-22. Terms are positive, so their sum is as good, plus its own rounding: a
chain of n additions n 2^-24. Old weights times decay are rounded once, and added once."""
import numpy as np
import pytest
import torch

from _tree import bf

gpu = pytest.mark.gpu
NAN = float("nan")


class Batch:
    """Rows of length `total` whose last `lens` tokens are queries; NaN in every slot that no query sees."""

    def __init__(self, total, lens, hq, hkv, seed, window=0, path=None, slots=None, queries=None, big=1.0):
        rng = np.random.default_rng(seed)
        self.total, self.hq, self.hkv, self.window = np.asarray(total), hq, hkv, window
        self.path = path
        self.n = np.array([len(x) for x in path]) if path is not None else np.asarray(lens)
        B = len(self.total)
        self.qsl = np.concatenate([[0], np.cumsum(lens)])
        T = int(self.qsl[-1])
        last = -(-self.total // 16)
        width = max(1, int(last.max()))
        self.slots = slots or width * 16
        P = int(last.sum()) + 2
        ids = rng.permutation(P)
        self.bt = np.full((B, width), -1, np.int64)
        kc = np.full((P, hkv, 16, 64), np.nan)
        at = 0
        for r in range(B):
            lo = max(0, self.total[r] - self.n[r] - window + 1) if window > 0 else 0
            first = lo // 16 if self.n[r] else last[r]  # pages before it are gone
            for j in range(first, last[r]):
                self.bt[r, j] = ids[at]
                at += 1
            pos = np.arange(lo, self.total[r]) if self.n[r] else np.zeros(0, np.int64)
            kc[self.bt[r, pos // 16], :, pos % 16] = rng.standard_normal((len(pos), hkv, 64))
        (self.kt, self.k), (self.qt, self.q) = bf(kc), bf(rng.standard_normal((T, hq, 64)) * big)
        self.lse = (np.log(np.maximum(np.repeat(self.total, lens), 1))[:, None] + 0.5
                    + 0.3 * rng.standard_normal((T, hq))).astype(np.float32)
        self.old = (rng.random((B, hkv, self.slots)) * 3).astype(np.float32)

    def reference(self, scale, decay):
        """New weights, and how far each may be off."""
        decay = float(np.float32(decay))  # what the call takes is a float
        out = self.old.astype(np.float64)
        bound = np.zeros_like(out)
        g = self.hq // self.hkv
        for r in range(len(self.total)):
            S, n = int(self.total[r]), int(self.n[r])
            if n == 0:
                continue
            C = S - n
            node = np.asarray(self.path[r]) if self.path is not None else np.arange(n)
            sums, terms = np.zeros((self.hkv, S)), np.zeros(S)
            lo = max(0, C - self.window + 1) if self.window > 0 else 0
            key = np.arange(lo, S)
            k = self.k[self.bt[r, key // 16], :, key % 16]  # [keys, hkv, 64]
            for i in range(n):
                t = int(self.qsl[r]) + int(node[i])
                sees = key <= C + i
                if self.window > 0:
                    sees &= C + i - key < self.window
                for h in range(self.hkv):
                    x = scale * k[:, h] @ self.q[t, h * g:(h + 1) * g].T - self.lse[t, h * g:(h + 1) * g].astype(np.float64)
                    e = np.where(np.isneginf(self.lse[t, h * g:(h + 1) * g]), 0.0, np.exp(x)).sum(1)
                    sums[h, lo:] += np.where(sees, e, 0)
                terms[lo:] += g * sees
            keep = np.where(np.arange(S) < C, decay, 0.0) * self.old[r, :, :S] if decay else np.zeros((self.hkv, S))
            out[r, :, :S] = keep + sums
            bound[r, :, :S] = sums * (2.5e-5 + terms * 2.0 ** -24) + 2 * 2.0 ** -24 * (keep + sums) + 1e-37
        return out, bound

    def run(self, scale=0.125, decay=1.0, want_status=0, ws=None):
        from paper_2608_22167_gb300 import mcpu

        i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()  # noqa: E731
        q, kc, bt, sl = self.qt.cuda(), self.kt.cuda(), i32(self.bt), i32(self.total)
        w = torch.from_numpy(self.old.copy()).cuda()
        ws = mcpu.new_weights_workspace(mcpu.dims(q, kc, bt, sl)) if ws is None else ws
        path = path_len = None
        if self.path is not None:
            most = max([len(x) for x in self.path] + [1])
            path = i32([list(x) + [-7] * (most - len(x)) for x in self.path])
            path_len = i32(self.n)
        mcpu.mcpu_accumulate_weights(q, torch.from_numpy(self.lse).cuda(), kc, bt, sl, i32(self.qsl), self.window,
                                     scale, decay, w, ws, query_path=path, path_len=path_len)
        assert mcpu.mcpu_read_device_status(ws)[1] == want_status
        return w

    def check(self, scale=0.125, decay=1.0):
        got = self.run(scale, decay).double().cpu().numpy()
        want, bound = self.reference(scale, decay)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        ok = ~np.isnan(want)
        worst = np.max(np.abs(got - want)[ok] - bound[ok], initial=-1.0)
        assert worst <= 0, f"off by {np.max((np.abs(got - want) / np.maximum(bound, 1e-300))[ok]):.2f} of the bound"
        return got


HEADS = [(8, 1), (8, 8), (4, 2), (16, 4), (16, 2), (64, 8)]


@gpu
@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("decay", [1.0, 0.75, 0.0])
def test_single_tokens(hq, hkv, decay):
    Batch([1, 2, 15, 16, 17, 100, 255, 256, 257, 700], [1] * 10, hq, hkv, seed=hq + hkv).check(decay=decay)


@gpu
@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("window", [0, 1, 16, 100, 1000])
def test_chunks(hq, hkv, window):
    total = [1, 40, 33, 300, 129, 600, 513, 700]
    lens = [1, 40, 0, 17, 128, 300, 2, 33]
    Batch(total, lens, hq, hkv, seed=7 * hq + hkv + window, window=window).check(decay=0.5 if window == 16 else 1.0)


@gpu
@pytest.mark.parametrize("g", [1, 2, 4, 8])
def test_long_chunks(g):
    # many query blocks per key, keys before, at and behind the diagonal
    Batch([1500, 2300, 64], [1500, 900, 64], 2 * g, 2, seed=g).check()


@gpu
@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("hq,hkv", [(64, 8), (8, 8), (4, 2)])
def test_chosen_queries(hq, hkv, window):
    lens = [1, 9, 28, 40, 20, 33, 4]
    path = [[0], [0, 3, 8], list(range(0, 28, 3)), [], [5, 5, 2], list(range(33)), [3]]
    total = [1, 60, 300, 90, 17, 33, 1000]
    b = Batch(total, lens, hq, hkv, seed=3, window=window, path=path)
    b.check(decay=0.9)
    b.check(decay=0.0)


@gpu
def test_long_rows_and_few():
    Batch([40000], [3], 16, 2, seed=1).check()
    Batch([9000, 70, 20011], [1, 70, 200], 8, 2, seed=2).check()


@gpu
def test_many_rows():
    rng = np.random.default_rng(4)
    lens = rng.integers(0, 5, 700)
    Batch(lens + rng.integers(0, 90, 700), lens, 8, 1, seed=5).check()


@gpu
def test_weight_rows_shorter_than_the_table():
    b = Batch([30, 60, 45], [2, 1, 45], 8, 2, seed=6, slots=61)
    b.check()
    b = Batch([30, 62, 45], [2, 1, 45], 8, 2, seed=6, slots=61)
    got = b.run(want_status=2).double().cpu().numpy()
    assert np.array_equal(got[1], b.old[1].astype(np.float64))  # does not fit: left alone


@gpu
def test_first_decode_without_old_weights_reads_none():
    b = Batch([50, 300], [3, 1], 8, 2, seed=8)
    b.old[:] = NAN
    got = b.run(decay=0.0).double().cpu().numpy()
    assert np.all(np.isfinite(got[0, :, :50])) and np.all(np.isfinite(got[1, :, :300]))
    assert np.all(np.isnan(got[0, :, 50:]))
    got = b.run(decay=1.0).double().cpu().numpy()  # new slots do not read theirs
    assert np.all(np.isfinite(got[0, :, 47:50])) and np.all(np.isnan(got[0, :, :47]))


@gpu
def test_queries_that_saw_nothing_and_nan():
    b = Batch([200, 90], [5, 90], 8, 2, seed=9)
    b.lse[2, 3] = -np.inf
    b.lse[7, :] = np.inf
    b.check()
    # a NaN in a key reaches that key's weights, in a query those of the keys that see it
    c = Batch([200, 90], [5, 90], 8, 2, seed=9)
    page, slot = c.bt[1, 20 // 16], 20 % 16
    c.k[page, 1, slot, 5] = NAN
    c.kt[page, 1, slot, 5] = NAN
    c.q[2, 0, 0] = NAN
    c.qt[2, 0, 0] = NAN
    got = c.check()
    assert np.isnan(got[1, 1, 20]) and not np.isnan(got[1, 0, 20]) and not np.isnan(got[1, 1, 21])
    assert np.all(np.isnan(got[0, 0, :198])) and np.all(np.isfinite(got[0, 0, 198:200]))


@gpu
def test_large_scores():
    b = Batch([500], [20], 8, 2, seed=10, big=30.0)
    # log-sum-exps that belong to the scores, so that weights are between 0 and 1
    for i in range(20):
        k = b.k[b.bt[0, np.arange(481 + i) // 16], :, np.arange(481 + i) % 16]
        for u in range(8):
            x = 0.125 * k[:, u // 4] @ b.q[i, u]
            b.lse[i, u] = x.max() + np.log(np.exp(x - x.max()).sum())
    got = b.run().double().cpu().numpy()
    want, _ = b.reference(0.125, 1.0)
    # the exponent is a difference of values up to 150: 64 2^-24 of a sum of 30 5 at most, and 150 2^-23
    assert np.max(np.abs(got - want) / (np.abs(want) + 1e-30)) <= 64 * 150 * 2.0 ** -24 + 300 * 2.0 ** -24


@gpu
def test_bad_rows_and_pages():
    from paper_2608_22167_gb300 import mcpu

    b = Batch([100, 300, 50, 64], [1, 40, 2, 1], 8, 2, seed=11)
    want, bound = b.reference(0.125, 1.0)
    lost = b.bt[1, 7]
    b.bt[1, 7] = 10 ** 6
    b.bt[3, 0] = -1
    got = b.run(want_status=1).double().cpu().numpy()
    keys = np.ones(want.shape, bool)
    keys[1, :, 112:128] = keys[3, :, 0:16] = False
    assert np.all((np.abs(got - want) <= bound)[keys]) and np.array_equal(got[~keys], b.old[~keys].astype(np.float64))
    b.bt[1, 7], b.bt[3, 0] = lost, b.bt[3, 1]
    for path in ([[0], [40], [1], [0]], [[0], [-1], [1], [0]]):
        b.path, b.n = path, np.array([1, 1, 1, 1])
        got = b.run(want_status=2).cpu().numpy()
        assert np.array_equal(got[1], b.old[1]) and not np.array_equal(got[0], b.old[0])
    b.path, b.n = None, np.array([1, 40, 2, 1])
    b.total = np.array([100, 39, 50, 64])
    assert np.array_equal(b.run(want_status=2).cpu().numpy()[1], b.old[1])
    b.total = np.array([100, 300, 50, 64])
    b.qsl = b.qsl + 1
    assert np.array_equal(b.run(want_status=2).cpu().numpy(), b.old)
    ws = mcpu.new_weights_workspace(mcpu.Dims(1, 1, 1, 1, 1, 1, 64, 16))
    b.qsl = b.qsl - 1
    b.run(ws=ws)


@gpu
def test_same_bits_every_time_and_in_graphs():
    from paper_2608_22167_gb300 import mcpu

    b = Batch([3000, 500, 1200, 90], [700, 1, 64, 90], 16, 2, seed=12)
    first = b.run()
    for _ in range(3):
        assert torch.equal(b.run(), first)
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()  # noqa: E731
    q, kc, bt, sl, qsl = b.qt.cuda(), b.kt.cuda(), i32(b.bt), i32(b.total), i32(b.qsl)
    w, lse = torch.from_numpy(b.old).cuda(), torch.from_numpy(b.lse).cuda()
    ws = mcpu.new_weights_workspace(mcpu.dims(q, kc, bt, sl))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mcpu.mcpu_accumulate_weights(q, lse, kc, bt, sl, qsl, 0, 0.125, 1.0, w, ws)
    side = torch.cuda.Stream()
    for lens in ([700, 1, 64, 90], [1, 700, 90, 64]):
        c = Batch([3000, 900, 1200, 90], lens, 16, 2, seed=13)
        kc[:] = 0
        kc[: len(c.kt)] = c.kt.cuda()[: len(kc)]
        c.bt[c.bt >= len(kc)] = 0
        c.kt = kc.cpu()
        c.k = c.kt.double().numpy()
        q.copy_(c.qt), bt.fill_(-1), bt[:, : c.bt.shape[1]].copy_(i32(c.bt)), sl.copy_(i32(c.total))
        qsl.copy_(i32(c.qsl)), lse.copy_(torch.from_numpy(c.lse)), w.copy_(torch.from_numpy(c.old))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        side.synchronize()
        got = w.double().cpu().numpy()
        want, bound = c.reference(0.125, 1.0)
        ok = ~np.isnan(want)
        assert np.all(np.abs(got - want)[ok] <= bound[ok])


@gpu
def test_offsets_past_32_bits():
    """A pool of more than 4 GiB, and weights whose rows begin past 2^31 elements."""
    from paper_2608_22167_gb300 import mcpu

    b = Batch([40, 100], [1, 3], 8, 2, seed=14)
    pages = 2 ** 32 // (2 * 2048) + 100
    kc = torch.empty(pages, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    kc[pages - len(b.kt):] = b.kt.cuda()
    slots = 600_000_000
    w = torch.empty(2, 2, slots, device="cuda")
    w[:, :, : b.slots] = torch.from_numpy(b.old).cuda()
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()  # noqa: E731
    q, bt, sl = b.qt.cuda(), i32(np.where(b.bt >= 0, b.bt + pages - len(b.kt), -1)), i32(b.total)
    ws = mcpu.new_weights_workspace(mcpu.dims(q, kc, bt, sl))
    mcpu.mcpu_accumulate_weights(q, torch.from_numpy(b.lse).cuda(), kc, bt, sl, i32(b.qsl), 0, 0.125, 1.0, w, ws)
    assert mcpu.mcpu_read_device_status(ws)[1] == 0
    want, bound = b.reference(0.125, 1.0)
    assert np.all(np.abs(w[:, :, : b.slots].double().cpu().numpy() - want) <= bound)


@gpu
def test_a_row_and_a_window_of_more_than_2_30_keys():
    """Slot + window pass 2^31. The keys are zeros, so that a head's weight of a key it sees is exp(-lse) = 1 exactly."""
    from paper_2608_22167_gb300 import mcpu

    S, W, missing = 1_100_000_000, 1_080_000_000, 1_090_000_000 // 16
    q = torch.ones(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    kc = torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16, device="cuda")
    table = torch.ones(1, S // 16, dtype=torch.int32, device="cuda")
    table[0, missing] = 7  # no such page
    w = torch.zeros(1, 1, S, device="cuda")
    lens = torch.tensor([S], dtype=torch.int32, device="cuda")
    qsl = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    ws = mcpu.new_weights_workspace(mcpu.dims(q, kc, table, lens))
    mcpu.mcpu_accumulate_weights(q, torch.zeros(1, 1, device="cuda"), kc, table, lens, qsl, W, 0.125, 1.0, w, ws)
    assert mcpu.mcpu_read_device_status(ws)[1] == mcpu.STATUS_BAD_PAGE
    w = w.view(-1)
    first = S - W  # the query's position is S - 1
    assert not w[:first].any() and not w[16 * missing : 16 * missing + 16].any()
    assert int((w == 1).sum()) == W - 16


@gpu
def test_weights_of_a_forward_call_sum_to_the_queries():
    """With the log-sum-exps of mcpu_paged_attention_forward a query's weights sum to one (less the sink's share), so
    a kv head's add up to its queries: 300 terms of 2.5e-5 relative, and an lse good to 1e-4."""
    from paper_2608_22167_gb300 import mcpu

    b = Batch([300, 150, 64], [100, 1, 64], 16, 2, seed=15)
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()  # noqa: E731
    q, kc, bt, sl, qsl = b.qt.cuda(), b.kt.cuda(), i32(b.bt), i32(b.total), i32(b.qsl)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    d = mcpu.dims(q, kc, bt, sl)
    mcpu.mcpu_paged_attention_forward(q, kc, kc, bt, sl, qsl, 0, 0.125, out, lse, mcpu.new_workspace(d))
    w = torch.zeros(3, 2, b.slots, device="cuda")
    ws = mcpu.new_weights_workspace(d)
    mcpu.mcpu_accumulate_weights(q, lse, kc, bt, sl, qsl, 0, 0.125, 1.0, w, ws)
    want = torch.tensor([100, 1, 64.0], device="cuda")[:, None] * 8
    assert torch.all((w.double().sum(2) - want).abs() <= 2e-4 * want)


@gpu
@pytest.mark.parametrize("window", [0, 700])
def test_paths_of_more_queries_than_the_step_has(window):
    """The same queries over and over: more blocks of them than the step's own queries fill, cut between the pieces."""
    rng = np.random.default_rng(16)
    path = [rng.integers(0, 40, 200).tolist(), [0, 0, 1]]
    Batch([5000, 90], [40, 2], 8, 1, seed=17, window=window, path=path).check(decay=0.5)


@gpu
@pytest.mark.parametrize("n", [1, 3, 17])
def test_keys_with_infinite_scores(n):
    """A key that every query scores -inf weighs nothing, one scored inf weighs inf: whatever the number of queries."""
    b = Batch([120, 40], [n, 1], 8, 1, seed=18)
    b.q[..., 0] = np.abs(b.q[..., 0]) + 1.0
    (b.qt, b.q) = bf(b.q)
    for key, value in ((5, -np.inf), (9, np.inf)):
        page, slot = b.bt[0, key // 16], key % 16
        b.k[page, 0, slot, 0] = b.kt[page, 0, slot, 0] = value
    got = b.run().double().cpu().numpy()
    want, bound = b.reference(0.125, 1.0)
    assert got[0, 0, 5] == b.old[0, 0, 5] and got[0, 0, 9] == np.inf
    finite = np.isfinite(want)
    assert np.all(np.abs(got[finite] - want[finite]) <= bound[finite])


def _args():
    from paper_2608_22167_gb300 import mcpu  # noqa: F401

    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t)  # noqa: E731
    bf16, f32 = torch.bfloat16, torch.float32
    return dict(q=z(4, 8, 64, t=bf16), lse=z(4, 8, t=f32), k_cache=z(5, 2, 16, 64, t=bf16), block_table=z(3, 6),
                seq_lens=z(3), query_start_loc=z(4), sliding_window=0, softmax_scale=0.125, decay=1.0,
                key_weights=z(3, 2, 96, t=f32), workspace=z(256, t=torch.uint8), query_path=z(3, 2), path_len=z(3),
                stream=None)


def test_binding_refuses_what_it_would_misread():
    from paper_2608_22167_gb300 import mcpu

    args = _args()
    with pytest.raises(ValueError, match="CUDA device"):  # the arguments as they are get as far as this
        mcpu.mcpu_accumulate_weights(**args)
    for key, x in args.items():
        if not torch.is_tensor(x) or x.dtype == torch.uint8:
            continue
        wrong = [x.double() if x.is_floating_point() else x.long(), torch.stack([x, x], -1)[..., 0]]
        if key in ("lse", "query_start_loc", "key_weights", "query_path", "path_len", "block_table"):
            wrong.append(x[:-1])
        for bad in wrong:
            with pytest.raises(ValueError, match="^(?!.*CUDA device)"):
                mcpu.mcpu_accumulate_weights(**dict(args, **{key: bad}))
    for bad in (dict(path_len=None), dict(query_path=None), dict(key_weights=torch.zeros(3, 3, 96))):
        with pytest.raises(ValueError, match="^(?!.*CUDA device)"):
            mcpu.mcpu_accumulate_weights(**dict(args, **bad))


def test_host_checks():
    from paper_2608_22167_gb300 import mcpu

    P, f = 1 << 20, mcpu._lib.mcpu_accumulate_weights
    dims = mcpu._pack_dims(3, 4, 6, 5, 8, 2, 64, 16)
    d = mcpu.Dims(3, 4, 6, 5, 8, 2, 64, 16)
    need = mcpu.mcpu_weights_workspace_size(d)
    assert need >= 256 and mcpu.mcpu_weights_workspace_size(mcpu.Dims(3, 4, 6, 5, 8, 3, 64, 16)) == 0
    ok = [P, P, P, P, P, P, P, 2, P, 0, 0.125, 1.0, dims, P, 96, P, need, None]
    empty = mcpu._pack_dims(0, 0, 6, 5, 8, 2, 64, 16)
    assert f(*[empty if i == 12 else x for i, x in enumerate(ok)]) == 0
    for i, bad in ((0, None), (0, P + 8), (1, None), (2, P + 8), (3, None), (4, P + 2), (5, None), (6, None), (7, -1),
                   (8, None), (10, 0.0), (10, float("nan")), (11, -0.1), (11, 1.5), (11, float("nan")), (12, None),
                   (13, None), (14, 0), (15, None), (15, P + 16), (12, mcpu._pack_dims(3, 4, 6, 0, 8, 2, 64, 16))):
        assert f(*[bad if k == i else x for k, x in enumerate(ok)]) == 1, (i, bad)
    assert f(*[need - 1 if k == 16 else x for k, x in enumerate(ok)]) == 3
    assert f(*[mcpu._pack_dims(3, 4, 6, 5, 8, 2, 128, 16) if k == 12 else x for k, x in enumerate(ok)]) == 2
    if not torch.cuda.is_available():
        assert f(*ok) == 4
