"""The calls of a tree-drafted round together: the cache and its pages after a
round are those of plain decoding, and greedy decoding with drafted trees
makes the tokens that greedy decoding token by token makes."""
import numpy as np
import pytest
import torch

gpu = pytest.mark.gpu


def test_tree_masks():
    from paper_2608_22167_gb300.tree_decode import tree_masks

    mask, depth = tree_masks([[-1, 0, 0, 2], [-1, -1] + list(range(1, 40))])
    assert mask.shape == (4 + 41, 2) and depth[:6].tolist() == [0, 1, 1, 2, 0, 0]
    assert mask[:4, 0].tolist() == [1, 3, 5, 13]
    full = mask.numpy().view(np.uint32).astype(np.uint64)
    bits = full[4:, 0] | full[4:, 1] << np.uint64(32)
    for i in range(2, 41):  # a chain hanging off node 1
        assert int(bits[i]) == sum(1 << j for j in range(1, i + 1))
    with pytest.raises(ValueError):
        tree_masks([[0]])


def test_accept_greedy():
    from paper_2608_22167_gb300.tree_decode import accept_greedy

    parents, tokens = [-1, 0, 0, 2, 3], [7, 1, 2, 5, 6]
    assert accept_greedy(parents, tokens, [2, 9, 5, 6, 4]) == ([0, 2, 3, 4], 4)
    assert accept_greedy(parents, tokens, [3, 9, 5, 6, 4]) == ([0], 3)


def _cache(model, rows, pages=400, width=40):
    from paper_2608_22167_gb300.tree_decode import PagedCache

    return PagedCache(len(model.o), rows, width, pages, model.hq, model.hkv)


def _feed(model, cache, chains):
    """Appends a chain of tokens to each row; the logits of all of them."""
    from paper_2608_22167_gb300.tree_decode import tree_masks

    lens = [len(c) for c in chains]
    mask, depth = tree_masks([list(range(-1, n - 1)) for n in lens])
    ctx = cache.seq_lens.clone()
    rep = torch.tensor(lens, device="cuda")
    qsl = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")
    cache.extend(ctx + rep.int())
    toks = torch.tensor([t for c in chains for t in c], device="cuda")
    return model.run(cache, toks, qsl, mask.cuda(), (ctx.repeat_interleave(rep) + depth.cuda()).int())


def _row(cache, r):
    """K and V of row r, every layer, by position."""
    n = int(cache.seq_lens[r])
    pos = torch.arange(n, device="cuda")
    page = cache.block_table[r].long()[pos // 16]
    return torch.stack([p[page, :, pos % 16] for p in cache.k + cache.v])


@gpu
def test_a_round_leaves_the_cache_of_plain_decoding():
    from paper_2608_22167_gb300.tree_decode import ToyModel, tree_masks

    model = ToyModel(seed=1)
    g = torch.Generator()
    g.manual_seed(3)
    rows, nodes = 5, 33
    draw = lambda n: torch.randint(0, model.vocab, (n,), generator=g).tolist()  # noqa: E731
    prompts = [draw(n) for n in (1, 15, 16, 47, 200)]
    tree, plain = _cache(model, rows), _cache(model, rows)
    _feed(model, tree, prompts)
    _feed(model, plain, prompts)
    parents = [[-1] + [int(torch.randint(max(-1, i - 4), i, (1,), generator=g)) for i in range(1, nodes)]
               for _ in range(rows)]
    tokens = [draw(nodes) for _ in range(rows)]
    mask, depth = tree_masks(parents)
    ctx = tree.seq_lens.clone()
    qsl = torch.arange(0, rows * nodes + 1, nodes, dtype=torch.int32, device="cuda")
    tree.extend(ctx + nodes)
    logits = model.run(tree, torch.tensor(tokens, device="cuda").flatten(), qsl, mask.cuda(),
                       (ctx.repeat_interleave(nodes) + depth.cuda()).int()).view(rows, nodes, -1)
    paths = []
    for r in range(rows):  # a random node's ancestors
        at, path = int(torch.randint(0, nodes, (1,), generator=g)), []
        while at >= 0:
            path.append(at)
            at = parents[r][at]
        paths.append(path[::-1])
    paths[2] = []  # nothing accepted
    most = max(map(len, paths))
    tree.keep(qsl, torch.tensor([p + [0] * (most - len(p)) for p in paths], dtype=torch.int32, device="cuda"),
              torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda"))
    tree.check()
    ref = _feed(model, plain, [[tokens[r][i] for i in paths[r]] for r in range(rows)])
    plain.check()
    assert tree.seq_lens.tolist() == plain.seq_lens.tolist() == [len(p) + len(q) for p, q in zip(prompts, paths)]
    assert int(tree.free_count) == int(plain.free_count)
    at = 0
    for r in range(rows):
        n = len(prompts[r])
        # layer 0's rows depend on the tokens only: bit for bit; layer 1's on rounded attention outputs
        a, b = _row(tree, r), _row(plain, r)
        assert torch.equal(a[:, :n], b[:, :n]) and torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])
        assert torch.allclose(a.float(), b.float(), atol=0.15)
        for i, node in enumerate(paths[r]):
            x, y = logits[r, node], ref[at + i]
            assert float((x - y).abs().max()) <= 0.05 * float(y.std()) + 0.05 * float(y.abs().max())
        at += len(paths[r])


@gpu
def test_greedy_trees_make_the_tokens_of_plain_decoding():
    from paper_2608_22167_gb300.tree_decode import ToyModel, generate

    model = ToyModel(seed=2)
    prompts, rows = 2, 6
    cache = _cache(model, rows)
    chains = [[1, 2, 3, 4, 5, 6, 7, 8, 9, 1, 2, 3, 4, 5, 6, 7, 8], [5] * 40] + [[] for _ in range(4)]
    _feed(model, cache, chains)
    cache.fork(torch.tensor([0, 1, 1, 0], dtype=torch.int32, device="cuda"),
               torch.tensor([2, 3, 4, 5], dtype=torch.int32, device="cuda"))
    cache.check()
    last = [3, 3, 4, 3, 5, 6]
    made = generate(model, cache, list(last), rounds=6, seed=5)
    assert max(len(m) for m in made) > 6  # some drafts were accepted
    full = [chains[i] + [t] for i, t in zip((0, 1, 0, 1, 1, 0), last)]
    plain = _cache(model, rows)
    logits = _feed(model, plain, [f + m[:-1] for f, m in zip(full, made)])
    plain.check()
    at = 0
    for f, m in zip(full, made):
        x = logits[at + len(f) - 1: at + len(f) + len(m) - 1]
        at += len(f) + len(m) - 1
        best = x.max(1).values
        got = x[torch.arange(len(m)), torch.tensor(m, device="cuda")]
        # the same tokens, but for ties within the rounding of a bf16 layer
        assert torch.all(got >= best - 0.05 * x.abs().max(1).values)
        assert (got == best).float().mean() > 0.9
    cache.drop(torch.arange(rows, device="cuda"))
    cache.check()
    assert int(cache.free_count) == 400 and not cache.page_refs.any() and bool((cache.block_table == -1).all())
    assert torch.equal(cache.free_pages.sort().values, torch.arange(400, dtype=torch.int32, device="cuda"))


@gpu
def test_the_example_runs(capsys):
    from paper_2608_22167_gb300 import tree_decode

    tree_decode.main()
    assert "tokens" in capsys.readouterr().out


@gpu
def test_a_captured_round_replays():
    from paper_2608_22167_gb300 import mcpu
    from paper_2608_22167_gb300.tree_decode import ToyModel, tree_masks

    model = ToyModel(seed=4)
    cache = _cache(model, 3)
    _feed(model, cache, [[1, 2, 3], [4] * 30, [5] * 16])
    nodes = 9
    mask, depth = tree_masks([[-1, 0, 0, 1, 1, 2, 3, 3, 5]] * 3)
    mask, depth = mask.cuda(), depth.cuda()
    qsl = torch.arange(0, 3 * nodes + 1, nodes, dtype=torch.int32, device="cuda")
    tokens = torch.arange(3 * nodes, device="cuda") % model.vocab
    path = torch.tensor([[0, 2, 5], [0, 1, 4], [0, 0, 0]], dtype=torch.int32, device="cuda")
    taken = torch.tensor([3, 2, 1], dtype=torch.int32, device="cuda")
    x = model.embed[tokens]
    h = (x.float() @ model.qkv[0].float()).to(torch.bfloat16)
    q, k, v = (t.unflatten(1, (-1, 64)) for t in h.split([512, 128, 128], dim=1))
    q_out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    out, lse = torch.empty_like(q_out), torch.empty(q.shape[:2], device="cuda")
    ctx = cache.seq_lens.clone()
    want, pos = torch.empty_like(ctx), torch.empty(3 * nodes, dtype=torch.int32, device="cuda")

    def round_():
        torch.add(cache.seq_lens, nodes, out=want)
        pos.view(3, nodes).copy_(cache.seq_lens[:, None] + depth.view(3, nodes))
        cache.extend(want)
        for layer in range(2):
            cache.append(layer, q, k, v, model.norm[0][0], model.norm[0][1], 1e-6, model.cos_sin, qsl, pos, q_out=q_out)
            cache.attend(layer, q_out, qsl, mask, pos, sliding_window=20, out=out, lse=lse)
        cache.keep(qsl, path, taken)

    def state():
        return [t.clone() for t in (out, lse, cache.seq_lens, cache.free_count, cache.page_refs)]

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        round_()
    torch.cuda.synchronize()
    eager = []
    for _ in range(3):
        round_()
        eager.append(state())
    cache.seq_lens.copy_(ctx + taken)  # back to the state after the first round
    cache._release(cache.seq_lens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        round_()
    for want_state in eager:
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(state(), want_state):
            assert torch.equal(a, b)
    assert mcpu.mcpu_read_device_status(cache.workspace) == (0, 0)


@gpu
def test_pages_far_into_large_pools():
    # byte offsets past 32 bits: 20000 pages of 128 kv heads are 5.2 GB a pool
    from paper_2608_22167_gb300 import mcpu

    hkv, pages = 128, 20000
    pools = [torch.empty(pages, hkv, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    bt, sl, qsl = i32([[19999, 3, 19500, 19001]]), i32([50]), i32([0, 20])
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    for p in pools:
        p[bt[0].long()] = randn(4, hkv, 16, 64)
    q, k, v = randn(20, hkv, 64), randn(20, hkv, 64), randn(20, hkv, 64)
    w, tab, status = torch.ones(64, device="cuda"), torch.zeros(64, 64, device="cuda"), i32([0])
    tab[:, :32] = 1  # no rotation
    q_out = torch.empty_like(q)
    mcpu.mcpu_norm_rope_kv_append(q, k, v, w, w, 0.0, None, tab, q_out, *pools, bt, sl, qsl, status)
    slot = torch.arange(30, 50, device="cuda")
    assert torch.equal(pools[1][bt[0, slot // 16].long(), :, slot % 16], v)
    norm = lambda x: x.double() / x.double().square().mean(-1, keepdim=True).sqrt()  # noqa: E731
    assert (pools[0][bt[0, slot // 16].long(), :, slot % 16].double() - norm(k)).abs().max() <= 2.0 ** -6
    ws = mcpu.new_tree_workspace(mcpu.dims(q, pools[0], bt, sl))
    out, lse = torch.empty_like(q), torch.empty(20, hkv, device="cuda")
    mask = i32([[(1 << i + 1) - 1] for i in range(20)])
    mcpu.mcpu_tree_attention_forward(q_out, *pools, bt, sl, qsl, mask, None, 0, 0.125, out, lse, ws)
    pos = torch.arange(50, device="cuda")
    kk, vv = (p[bt[0, pos // 16].long(), :, pos % 16].double() for p in pools)
    x = torch.einsum("thd,jhd->thj", q_out.double(), kk) * 0.125
    x = x.masked_fill(pos[None, None] > (30 + torch.arange(20, device="cuda"))[:, None, None], -torch.inf)
    ref = torch.einsum("thj,jhd->thd", x.softmax(-1), vv)
    mag = torch.einsum("thj,jhd->thd", x.softmax(-1), vv.abs())
    assert ((out.double() - ref).abs() <= 1.01 * 2.0 ** -8 * (mag + ref.abs()) + 1e-6).all()
    assert (lse.double() - x.logsumexp(-1)).abs().max() <= 1e-4
    lst = mcpu.PoolList(pools)
    new = i32([0])
    mcpu.mcpu_compact_kv(lst, bt, sl, qsl, i32([[1, 18, 19]]), i32([3]), new, status)
    kept = torch.tensor([31, 48, 49], device="cuda")
    slot = torch.arange(30, 33, device="cuda")
    assert torch.equal(pools[1][bt[0, slot // 16].long(), :, slot % 16], vv[kept].to(torch.bfloat16))
    mcpu.mcpu_copy_pages(lst, i32([19999, 3]), i32([5, 19998]), status)
    for p in pools:
        assert torch.equal(p[5], p[19999]) and torch.equal(p[19998], p[3])
    assert int(new) == 33 and int(status) == 0 and mcpu.mcpu_read_device_status(ws) == (0, 0)


@gpu
@pytest.mark.parametrize("window", [1, 40, 64])
def test_rounds_in_a_window_need_the_windows_pages_only(window):
    # the same rounds over a cache that keeps every page and one with room for the windows alone
    from paper_2608_22167_gb300.tree_decode import PagedCache, rope_table, tree_masks

    rows, nodes, hq, hkv = 5, 20, 8, 2
    caches = [PagedCache(1, rows, 40, 240, hq, hkv), PagedCache(1, rows, 40, 16 * rows, hq, hkv, sliding_window=window)]
    tab, w = rope_table(800), torch.ones(64, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(window)
    lens = [0] * rows
    for n in [200, 1, 17] + [nodes] * 10:
        # a chain, or one of 14 nodes with others hanging off it
        mask, depth = tree_masks([[i - 1 if i < 14 or n > nodes else i - 12 for i in range(n)]] * rows)
        qsl = torch.arange(0, rows * n + 1, n, dtype=torch.int32, device="cuda")
        pos = (torch.tensor(lens).repeat_interleave(n) + depth).int().cuda()
        x = torch.randn(rows * n, hq + 2 * hkv, 64, generator=g, device="cuda", dtype=torch.bfloat16)
        path = list(range(n if n > nodes else min(n, 14)))  # one row keeps nothing
        taken = [0 if r == 3 else len(path) - (r == 2 and n > 1) for r in range(rows)]
        outs = []
        for cache in caches:
            cache.extend(torch.tensor(lens, device="cuda") + n)
            q = cache.append(0, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], w, w, 1e-6, tab, qsl, pos)
            outs.append(cache.attend(0, q, qsl, mask.cuda(), pos, sliding_window=window))
            cache.keep(qsl, torch.tensor([path] * rows, dtype=torch.int32, device="cuda"),
                       torch.tensor(taken, dtype=torch.int32, device="cuda"))
            cache.check()
        lens = [a + b for a, b in zip(lens, taken)]
        assert caches[1].seq_lens.tolist() == lens
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
        table = caches[1].block_table
        assert (table >= 0).sum(1).tolist() == [-(-s // 16) - max(0, s - window + 1) // 16 for s in lens]
        assert int(caches[1].free_count) == 16 * rows - table[table >= 0].unique().numel()
        if n == 17:  # a sample of row 0 in place of row 4
            for cache in caches:
                cache.drop(torch.tensor([4], device="cuda"))
                cache.fork(torch.tensor([0], dtype=torch.int32, device="cuda"),
                           torch.tensor([4], dtype=torch.int32, device="cuda"))
                cache.check()
            lens[4] = lens[0]
    assert sum(-(-s // 16) for s in lens) > 16 * rows


@pytest.mark.parametrize("window", [1, 2, 5, 31, 32, 33, 100])
def test_tree_masks_in_a_window(window):
    from paper_2608_22167_gb300.tree_decode import tree_masks

    rng = np.random.default_rng(window)
    parents = [list(range(-1, 69)), [-1] + [int(rng.integers(max(-1, i - 3), i)) for i in range(1, 80)], [-1, -1, 0]]
    mask, depth = tree_masks(parents, window)
    plain, same_depth = tree_masks(parents)
    assert torch.equal(depth, same_depth) and mask.shape == plain.shape
    bits = mask.numpy().view(np.uint32)
    t = 0
    for parent in parents:
        for i in range(len(parent)):
            want, at = set(), i
            while at >= 0 and len(want) < window:  # one level up, one position back
                want.add(at)
                at = parent[at]
            assert {n for n in range(32 * mask.shape[1]) if bits[t, n // 32] >> np.uint32(n % 32) & 1} == want
            t += 1
    if window > int(depth.max()):
        assert torch.equal(mask, plain)


@gpu
@pytest.mark.parametrize("window", [1, 17, 128])
def test_a_chain_deeper_than_its_window_is_a_windowed_chunk(window):
    # prompts fed as chains, the framework's plain windowed forward beside
    from paper_2608_22167_gb300 import mcpu
    from paper_2608_22167_gb300.tree_decode import PagedCache, tree_masks

    lens, ctx, hq, hkv = [200, 31, 140], [0, 55, 300], 16, 2
    cache = PagedCache(1, 3, 40, 100, hq, hkv, sliding_window=window)
    g = torch.Generator(device="cuda")
    g.manual_seed(window)
    cache.extend(torch.tensor([c + n for c, n in zip(ctx, lens)], device="cuda"))
    for p in cache.k + cache.v:
        p.normal_(generator=g)
    mask, depth = tree_masks([list(range(-1, n - 1)) for n in lens], window)
    pos = (torch.tensor(ctx).repeat_interleave(torch.tensor(lens)) + depth).int().cuda()
    qsl = torch.tensor([0, 200, 231, 371], dtype=torch.int32, device="cuda")
    q = torch.randn(371, hq, 64, generator=g, device="cuda", dtype=torch.bfloat16)
    out, lse = cache.attend(0, q, qsl, mask.cuda(), pos)
    cache.check()
    ws = mcpu.new_workspace(mcpu.dims(q, cache.k[0], cache.block_table, cache.seq_lens))
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    mcpu.mcpu_paged_attention_forward(q, cache.k[0], cache.v[0], cache.block_table, cache.seq_lens, qsl, window, 0.125,
                                      o2, l2, ws)
    # both round each weight and the output to bf16 once: 2^-8 of a weighted mean of |v| <= 6, twice
    assert float((out.float() - o2.float()).abs().max()) <= 2 * 2 * 2.0 ** -8 * 6
    assert float((lse - l2).abs().max()) <= 1e-4
