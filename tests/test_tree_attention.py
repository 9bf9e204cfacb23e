"""Tree attention over the paged cache against a plain 64-bit implementation."""
import ctypes

import numpy as np
import pytest
import torch

from _tree import TreeBatch, ancestors, assert_tree_close, random_tree

gpu = pytest.mark.gpu


def _run(b, sinks=None, positions=True, ws=None):
    from paper_2608_22167_gb300 import mcpu

    d = b.device()
    dims = mcpu.dims(d["q"], d["kc"], d["bt"], d["sl"])
    ws = mcpu.new_tree_workspace(dims) if ws is None else ws
    out = torch.full_like(d["q"], float("nan"))
    lse = torch.full(d["q"].shape[:2], float("nan"), device="cuda")
    sk = None if sinks is None else torch.from_numpy(np.asarray(sinks, np.float32)).cuda()
    mcpu.mcpu_tree_attention_forward(d["q"], d["kc"], d["vc"], d["bt"], d["sl"], d["qsl"], d["mask"],
                                     d["pos"] if positions else None, b.window, b.scale, out, lse, ws, sinks=sk)
    return out, lse, ws, d


def _check(b, sinks=None, positions=True):
    from paper_2608_22167_gb300 import mcpu

    out, lse, ws, _ = _run(b, sinks, positions)
    assert mcpu.mcpu_read_device_status(ws) == (0, 0)
    assert_tree_close(out, lse, b.reference(None if sinks is None else np.asarray(sinks, np.float32).astype(np.float64)))


@gpu
@pytest.mark.parametrize("hq,hkv", [(8, 8), (4, 2), (8, 2), (16, 2), (64, 8)])
@pytest.mark.parametrize("window", [0, 1, 16, 37, 128])
def test_random_trees(hq, hkv, window):
    rng = np.random.default_rng(hq * 100 + window)
    ctx = np.concatenate([[0, 1, 15, 16, 17, 127, 128, 129], rng.integers(0, 700, 6)])
    lens = np.concatenate([[1, 3, 1, 16, 17, 2, 31, 33], rng.integers(1, 64, 6)])
    _check(TreeBatch(ctx, lens, hq, hkv, 7 + window, window=window))


@gpu
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 128, 200, 256])
def test_tree_sizes(n):
    ctx = [0, 5, 130, 253]
    _check(TreeBatch(ctx, [n, max(1, n - 1), n, 1], 16, 2, n, words=8 if n == 200 else None))


@gpu
@pytest.mark.parametrize("seed", range(12))
def test_random_batches(seed):
    rng = np.random.default_rng(900 + seed)
    hkv = int(rng.choice([1, 2, 3, 8]))
    hq = hkv * int(rng.choice([1, 2, 4, 8]))
    rows = int(rng.integers(1, 12))
    ctx = np.where(rng.random(rows) < 0.3, rng.integers(0, 3000, rows), rng.integers(0, 200, rows))
    lens = np.where(rng.random(rows) < 0.2, rng.integers(0, 257, rows), rng.integers(0, 40, rows))
    lens[0] = max(1, lens[0])
    b = TreeBatch(ctx, lens, hq, hkv, seed, window=int(rng.choice([0, 0, 5, 64, 500])))
    _check(b, sinks=rng.standard_normal(hq) if seed % 2 else None)


@gpu
def test_one_head_a_group_and_the_longest_tree():
    _check(TreeBatch([0, 77, 1500], [256, 255, 129], 2, 2, 13))
    _check(TreeBatch([900, 77], [256, 200], 8, 1, 14, window=100))


@gpu
@pytest.mark.parametrize("hq,hkv", [(64, 8), (8, 2), (2, 2)])
def test_sinks(hq, hkv):
    rng = np.random.default_rng(3)
    _check(TreeBatch([0, 40, 900], [9, 20, 40], hq, hkv, 11), sinks=rng.standard_normal(hq) * 1.5)
    _check(TreeBatch([0, 40, 900], [9, 20, 40], hq, hkv, 12, window=32), sinks=rng.standard_normal(hq) * 3)


@gpu
@pytest.mark.parametrize("ctx", [5000, 20001])
@pytest.mark.parametrize("n", [1, 16, 61])
def test_long_rows_are_split(ctx, n):
    _check(TreeBatch([ctx, 3], [n, 2], 16, 2, ctx + n))


@gpu
@pytest.mark.parametrize("ctx,n,window", [(756, 12, 0), (757, 12, 0), (5003, 32, 720), (5011, 32, 721), (5003, 32, 737)])
def test_the_longest_rows_that_are_not_split(ctx, n, window):
    # six blocks of 128 keys: 48 pages, or nodes and window and a page
    _check(TreeBatch([ctx, ctx - 700, ctx], [n, n, 1], 16, 2, ctx + window, window=window))


@gpu
def test_rows_without_nodes_and_many_rows():
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 4, 300)
    lens[:3] = 0
    _check(TreeBatch(rng.integers(0, 90, 300), lens, 8, 2, 21))


@gpu
@pytest.mark.parametrize("sinks", [False, True])
def test_masks_that_leave_nothing(sinks):
    # nodes that see no node, in rows without a context (nothing at all) and with one; a node nobody sees
    rng = np.random.default_rng(6)
    sees = []
    for n in (5, 5, 40):
        s, _ = ancestors(random_tree(n, rng))
        s[1] = False
        s[3] = False
        s[:, n - 1] = False
        sees.append(s)
    b = TreeBatch([0, 33, 0], [5, 5, 40], 8, 2, 31, sees=sees)
    for r, n in enumerate((5, 5, 40)):  # its K and V are not finite
        p = int(b.S[r]) - 1
        for t in (b.kt, b.vt):
            t[b.bt[r, p // 16], :, p % 16] = float("nan")
        b.k[b.bt[r, p // 16], :, p % 16] = np.nan
    _check(b, sinks=rng.standard_normal(8) if sinks else None)


@gpu
def test_arbitrary_masks_and_extra_words():
    # any bits: nodes that see later nodes, not themselves; bits past the row's nodes mean nothing
    rng = np.random.default_rng(8)
    sees = [rng.random((n, n)) < 0.4 for n in (7, 32, 50)]
    b = TreeBatch([10, 0, 200], [7, 32, 50], 16, 2, 41, sees=sees, words=4)
    full = b.mask.view(np.uint32).copy()
    row = np.repeat(np.arange(3), b.lens)
    for t in range(len(full)):
        for j in range(int(b.lens[row[t]]), 128):
            full[t, j // 32] |= np.uint32(1 << (j % 32))
    b.mask = full.view(np.int32)
    _check(b)


@gpu
def test_peaked_and_large_scores():
    b = TreeBatch([300, 1000], [20, 40], 16, 2, 51, big=12.0)
    from paper_2608_22167_gb300 import mcpu

    out, lse, ws, _ = _run(b)
    assert mcpu.mcpu_read_device_status(ws) == (0, 0)
    ro, rl, mag = b.reference()
    # scores reach 12 * 8 * a few: their fp32 sums are off by 64 * 2^-24 * sum |q k| * scale, which moves every
    # weight by that much
    ds = 64 * 2.0 ** -24 * 0.125 * 12 * 64 * 4
    got = out.double().cpu().numpy()
    assert np.all(np.abs(got - ro) <= 1.01 * 2.0 ** -8 * (mag + np.abs(ro)) + 2 * ds * mag + 1e-6)
    assert np.max(np.abs(lse.double().cpu().numpy() - rl)) <= 1e-4 + ds


@gpu
@pytest.mark.parametrize("window", [0, 700])
@pytest.mark.parametrize("at", [(394, 450), (460, 520), (511, 700), (0, 63), (64, 130), (890, 899)])
@pytest.mark.parametrize("levels", [(0, 10, 16), (0, 20, 60), (0, 90, 110), (0, 200, 240), (0, 240, 0), (240, 0, 100)])
def test_scores_that_leap(levels, at, window):
    # keys from at[0] and at[1] on score level / 2 higher (nats; level / 8, or falling, in other rows of a warp): the
    # running reference is far too low in either half of a block, by up to 2^170
    b = TreeBatch([900, 903], [20, 5], 16, 2, 71, window=window)
    q, k = b.qt.clone(), b.kt.clone()
    q[:, :, 0] = torch.tensor([4.0, 1.0, -4.0, 0.0]).repeat(7)[: q.shape[0], None]
    for r in range(2):
        for p in range(max(0, int(b.ctx[r]) - window + 1) if window else 0, int(b.ctx[r])):
            k[b.bt[r, p // 16], :, p % 16, 0] = float(levels[sum(p >= x for x in at)])
    b.qt, b.q, b.kt, b.k = q, q.double().numpy(), k, k.double().numpy()
    from paper_2608_22167_gb300 import mcpu

    out, lse, ws, _ = _run(b)
    assert mcpu.mcpu_read_device_status(ws) == (0, 0)
    ro, rl, mag = b.reference()
    # |q k| sums to at most 4 * 240 + 64 * 4 * 4; the reference and lse are fp32 numbers of up to 2^8
    ds = 64 * 2.0 ** -24 * 0.125 * (4 * 240 + 64 * 16) + 2.0 ** -15
    got = out.double().cpu().numpy()
    assert np.all(np.abs(got - ro) <= 1.01 * 2.0 ** -8 * (mag + np.abs(ro)) + 2 * ds * mag + 1e-6)
    assert np.max(np.abs(lse.double().cpu().numpy() - rl)) <= 1e-4 + ds


@gpu
def test_positions_outside_the_tree_count_as_the_nearest_inside():
    b = TreeBatch([50, 80], [6, 9], 8, 2, 61, window=20)
    b.positions = b.positions + np.where(np.arange(15) % 2, 1000, -1000)
    _check(b)


@gpu
def test_same_bits_again_and_on_another_stream():
    from paper_2608_22167_gb300 import mcpu

    b = TreeBatch([4000, 10, 777], [30, 5, 17], 64, 8, 71)
    o1, l1, ws, d = _run(b)
    o2, l2, _, _ = _run(b, ws=ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o3, l3, _, _ = _run(b, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(o1, o2) and torch.equal(l1, l2) and torch.equal(o1, o3) and torch.equal(l1, l3)
    assert mcpu.mcpu_read_device_status(ws) == (0, 0)


@gpu
def test_a_causal_chunk_is_a_tree():
    # a chain of nodes is the append rows of the plain forward
    from paper_2608_22167_gb300 import mcpu

    lens = [1, 40, 7]
    b = TreeBatch([100, 333, 0], lens, 64, 8, 81, sees=[np.tril(np.ones((n, n), bool)) for n in lens])
    out, lse, ws, d = _run(b)
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    ws2 = mcpu.new_workspace(mcpu.dims(d["q"], d["kc"], d["bt"], d["sl"]))
    mcpu.mcpu_paged_attention_forward(d["q"], d["kc"], d["vc"], d["bt"], d["sl"], d["qsl"], 0, b.scale, o2, l2, ws2)
    ref = b.reference()
    assert_tree_close(out, lse, ref)
    assert_tree_close(o2, l2, ref)


@gpu
def test_graph_replay_follows_new_lengths_and_masks():
    from paper_2608_22167_gb300 import mcpu

    lens = [20, 3, 33]
    b = TreeBatch([900, 64, 15], lens, 16, 2, 91)
    c = TreeBatch([40, 700, 200], lens, 16, 2, 92)
    assert b.words == c.words
    d, e = b.device(), c.device()
    width = max(d["bt"].shape[1], e["bt"].shape[1])
    pages = max(d["kc"].shape[0], e["kc"].shape[0])

    def padded(x):
        bt = torch.full((3, width), -1, dtype=torch.int32, device="cuda")
        bt[:, :x["bt"].shape[1]] = x["bt"]
        kv = [torch.zeros(pages, *x[k].shape[1:], dtype=torch.bfloat16, device="cuda") for k in ("kc", "vc")]
        for a, k in zip(kv, ("kc", "vc")):
            a[:x[k].shape[0]] = x[k]
        return dict(x, bt=bt, kc=kv[0], vc=kv[1])

    d, e = padded(d), padded(e)
    ws = mcpu.new_tree_workspace(mcpu.dims(d["q"], d["kc"], d["bt"], d["sl"]))
    out, lse = torch.empty_like(d["q"]), torch.empty(d["q"].shape[:2], device="cuda")

    def call():
        mcpu.mcpu_tree_attention_forward(d["q"], d["kc"], d["vc"], d["bt"], d["sl"], d["qsl"], d["mask"], None, 0,
                                         0.125, out, lse, ws)

    call()
    assert_tree_close(out, lse, b.reference())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for k in d:
        d[k].copy_(e[k])
    out.fill_(float("nan"))
    g.replay()
    assert_tree_close(out, lse, c.reference())


@gpu
def test_device_errors():
    from paper_2608_22167_gb300 import mcpu

    # a row with more nodes than the mask has bits is skipped, the others are served
    b = TreeBatch([20, 30], [33, 5], 8, 2, 101, words=2)
    ref = b.reference()
    b.mask = b.mask[:, :1]
    out, lse, ws, _ = _run(b)
    assert mcpu.mcpu_read_device_status(ws)[0] == 10
    assert_tree_close(out[33:], lse[33:], tuple(x[33:] for x in ref))
    # a bad page of the context
    b = TreeBatch([40, 30], [3, 5], 8, 2, 102)
    b.bt[0, 1] = 10 ** 6
    out, lse, ws, _ = _run(b)
    assert mcpu.mcpu_read_device_status(ws)[0] == 5
    assert_tree_close(out[3:], lse[3:], tuple(x[3:] for x in _with_good_pages(b)))
    # more nodes than the length
    b = TreeBatch([40, 30], [3, 5], 8, 2, 103)
    ref = b.reference()
    b.S = np.array([2, 35])
    out, lse, ws, _ = _run(b)
    assert mcpu.mcpu_read_device_status(ws)[0] == 6
    assert_tree_close(out[3:], lse[3:], tuple(x[3:] for x in ref))


def _with_good_pages(b):
    """The reference with the pages outside the pool replaced by page 0."""
    b.bt = np.where(b.bt >= 10 ** 6, 0, b.bt)
    return b.reference()


def test_host_checks():
    from paper_2608_22167_gb300 import mcpu

    f = mcpu._lib.mcpu_tree_attention_forward
    d = mcpu.Dims(4, 9, 19, 34, 8, 2, 64, 16)
    P = 1 << 20  # an aligned address these calls never touch
    need = mcpu.mcpu_tree_workspace_size(d)
    assert need > 0 and need % 256 == 0
    assert mcpu.mcpu_tree_workspace_size(mcpu.Dims(4, 9, 19, 34, 8, 3, 64, 16)) == 0
    ok = dict(q=P, kc=P, vc=P, bt=P, sl=P, qsl=P, mask=P, words=1, pos=None, window=0, scale=0.125, sinks=None, dims=d,
              out=P, lse=P, ws=P, bytes=need)

    def call(**kw):
        a = dict(ok, **kw)
        return f(a["q"], a["kc"], a["vc"], a["bt"], a["sl"], a["qsl"], a["mask"], a["words"], a["pos"], a["window"],
                 a["scale"], a["sinks"], ctypes.byref(a["dims"]), a["out"], a["lse"], a["ws"], a["bytes"], None)

    for name in ("q", "kc", "vc", "bt", "sl", "qsl", "mask", "out", "lse", "ws"):
        assert call(**{name: None}) == 1, name
    for name in ("q", "kc", "vc", "out"):
        assert call(**{name: P + 8}) == 1, name
    assert call(mask=P + 2) == 1 and call(pos=P + 2) == 1 and call(sinks=P + 2) == 1 and call(ws=P + 16) == 1
    assert call(words=0) == 1 and call(words=9) == 1
    assert call(scale=0.0) == 1 and call(scale=float("nan")) == 1 and call(scale=float("inf")) == 1
    assert call(window=5) == 1  # a window needs positions
    assert call(bytes=need - 1) == 3
    assert call(dims=mcpu.Dims(4, 9, 19, 34, 8, 2, 128, 16)) == 2
    assert call(dims=mcpu.Dims(0, 0, 19, 34, 8, 2, 64, 16)) == 0  # nothing to do


@gpu
def test_blocks_given_up_halfway_are_the_same_every_time():
    # from some key on a row's scores lie 48 nats above all before: that block's first weights are stored before their
    # sum shows it, and the block is done anew over the same columns
    rng = np.random.default_rng(131)
    ctx = rng.integers(600, 1500, 40)
    b = TreeBatch(ctx, rng.integers(1, 17, 40), 16, 2, 131)
    q, k = b.qt.clone(), b.kt.clone()
    q[:, :, 0] = 4.0
    for r in range(40):
        at = int(rng.integers(256, ctx[r] - 129))
        for p in range(int(ctx[r])):
            k[b.bt[r, p // 16], :, p % 16, 0] = 96.0 if p >= at else 0.0
    b.qt, b.q, b.kt, b.k = q, q.double().numpy(), k, k.double().numpy()
    from paper_2608_22167_gb300 import mcpu

    out, lse, ws, _ = _run(b)
    ro, rl, mag = b.reference()
    # |q k| sums to at most 4 * 96 + 64 * 4 * 4; the reference and lse are fp32 numbers of up to 2^8
    ds = 64 * 2.0 ** -24 * 0.125 * (4 * 96 + 64 * 16) + 2.0 ** -15
    got = out.double().cpu().numpy()
    assert np.all(np.abs(got - ro) <= 1.01 * 2.0 ** -8 * (mag + np.abs(ro)) + 2 * ds * mag + 1e-6)
    assert np.max(np.abs(lse.double().cpu().numpy() - rl)) <= 1e-4 + ds
    for _ in range(20):
        again, lse2, _, _ = _run(b, ws=ws)
        assert torch.equal(again, out) and torch.equal(lse2, lse)
    assert mcpu.mcpu_read_device_status(ws) == (0, 0)


@gpu
@pytest.mark.parametrize("sinks", [False, True])
@pytest.mark.parametrize("ctx,window", [(70, 0), (400, 0), (6000, 0), (6000, 3000), (6000, 100)])
@pytest.mark.parametrize("what", ["q", "k", "node", "all k", "inf"])
def test_nan_reaches_what_sees_it_and_nothing_else(what, ctx, window, sinks):
    # the longer rows are cut into parts, the shorter ones are not: both give what the formula gives
    b = TreeBatch([ctx, 50, ctx], [9, 3, 20], 16, 2, 5 + ctx, window=window)
    rng = np.random.default_rng(ctx)
    if what == "q":
        b.qt[2, 3, 7] = b.qt[10, 15, 0] = float("nan")
    elif what == "node":  # seen by its descendants
        p = ctx + 1
        b.kt[b.bt[0, p // 16], 1, p % 16, 5] = float("nan")
    else:
        for p in (range(max(0, ctx - window + 1) if window else 0, ctx + 9) if what == "all k" else [ctx - 40]):
            b.kt[b.bt[0, p // 16], 0, p % 16, 3] = float("inf" if what == "inf" else "nan")
    b.q, b.k = b.qt.double().numpy(), b.kt.double().numpy()
    sk = rng.standard_normal(16).astype(np.float32) if sinks else None
    out, lse, ws, _ = _run(b, sk)
    from paper_2608_22167_gb300 import mcpu

    assert mcpu.mcpu_read_device_status(ws) == (0, 0)
    with np.errstate(invalid="ignore"):
        ro, rl, mag = b.reference(None if sk is None else sk.astype(np.float64))
    bad = np.isnan(rl)
    assert bad.any() and not bad.all() and np.array_equal(np.isnan(ro).all(2), bad)
    assert torch.isnan(out.cpu()[bad]).all() and torch.isnan(lse.cpu()[bad]).all()
    good = torch.from_numpy(~bad)
    assert_tree_close(out.cpu()[good], lse.cpu()[good], (ro[~bad], rl[~bad], mag[~bad]))


@gpu
@pytest.mark.parametrize("hq,hkv", [(16, 2), (2, 2)])
@pytest.mark.parametrize("ctx,n,window", [(600, 60, 64), (130, 6, 20), (50, 40, 1), (6000, 200, 1500), (6000, 256, 100)])
def test_keys_that_no_node_sees_may_hold_anything(ctx, n, window, hq, hkv):
    # positions that all lie past the context's end: the first keys of the first node's window are seen by none, and
    # whole pages of them may be missing
    b = TreeBatch([ctx, 3, ctx + 7], [n, 2, n], hq, hkv, ctx + n, window=window)
    rng = np.random.default_rng(n)
    for r in (0, 2):
        t = int(b.qsl[r])
        past = n // 2
        b.positions[t:t + n] = b.ctx[r] + rng.integers(past, n, n)
        b.positions[t + n // 3] = b.ctx[r] + past
        first = int(b.ctx[r]) + past - window + 1  # of the keys that are seen
        for p in range(max(0, int(b.ctx[r]) - window + 1), min(first, int(b.ctx[r]))):
            for x in (b.kt, b.vt):
                x[b.bt[r, p // 16], :, p % 16] = float("nan")
        b.bt[r, :max(0, min(first, int(b.ctx[r]))) // 16] = -1
    _check(b)


@gpu
def test_a_missing_page_that_a_node_sees_is_reported():
    from paper_2608_22167_gb300 import mcpu

    # keys from 560 on are seen; or no context key at all, and page 37 holds the first nodes
    for window, past, lost, code in ((50, 9, 34, 0), (50, 9, 35, 5), (3, 9, 36, 0), (3, 9, 37, 5)):
        b = TreeBatch([600], [30], 16, 2, 3, window=window)
        b.positions[:] = 600 + np.arange(30) % 20 + past
        b.bt[0, lost] = -1
        _, _, ws, _ = _run(b)
        assert mcpu.mcpu_read_device_status(ws)[0] == code
