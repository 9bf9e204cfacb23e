"""A drafted round whose end is decided on the device: verification, accumulated weights and eviction together, as
PagedCache runs them."""
import numpy as np
import pytest
import torch

from _verify import reference

gpu = pytest.mark.gpu
HQ, HKV, NODES = 8, 2, 12


def _cache(rows, layers=2, pages=300, width=24, **kw):
    from paper_2608_22167_gb300.tree_decode import PagedCache

    return PagedCache(layers, rows, width, pages, HQ, HKV, count_weights=True, **kw)


def _trees(rows, seed, vocab):
    g = torch.Generator()
    g.manual_seed(seed)
    parents = [[-1] + [int(torch.randint(max(0, i - 4), i, (1,), generator=g)) for i in range(1, NODES)]
               for _ in range(rows)]
    return parents, torch.randint(0, vocab, (rows, NODES), generator=g)


def _keys(cache, layer, r):
    """K of row r's slots [slots, heads, 64] in 64 bits."""
    at = torch.arange(int(cache.seq_lens[r]), device="cuda")
    page = cache.block_table[r].long()[at // 16]
    return cache.k[layer][page, :, at % 16].double()


def _step(cache, gen, ctx, lens, parents):
    """Appends trees with random q, k and v in every layer and attends; the qs, and query_start_loc."""
    from paper_2608_22167_gb300.tree_decode import rope_table, tree_masks

    mask, depth = tree_masks(parents)
    qsl = torch.tensor([0] + np.cumsum(lens).tolist(), dtype=torch.int32, device="cuda")
    rep = torch.tensor(lens, device="cuda")
    pos = ((torch.tensor(ctx, device="cuda") + cache.evicted).repeat_interleave(rep) + depth.cuda()).int()
    cache.extend(torch.tensor([c + n for c, n in zip(ctx, lens)], device="cuda"))
    ones, tab = torch.ones(64, device="cuda"), rope_table(2000)
    qs = []
    for layer in range(len(cache.k)):
        x = torch.randn(sum(lens), HQ + 2 * HKV, 64, generator=gen, device="cuda", dtype=torch.bfloat16)
        q = cache.append(layer, x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], ones, ones, 1e-6, tab, qsl, pos)
        cache.attend(layer, q, qsl, mask.cuda(), pos)
        qs.append(q)
    return qs, qsl


@gpu
def test_weights_of_a_round_are_those_of_the_accepted_chain():
    """After prompts and a round, every key's weight is the softmax weight that the accepted queries gave it: a term
    is good to 2.2e-5 (the key weights' own tolerance) and 1e-4 of the log-sum-exp of tree attention."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    rows, lens = 3, [40, 90, 17]
    cache = _cache(rows)
    chains = [list(range(-1, n - 1)) for n in lens]
    want = [torch.zeros(rows, HKV, cache.key_weights.shape[3], dtype=torch.float64, device="cuda") for _ in range(2)]

    def add(qs, qsl, ctx, paths, decay):
        for layer, q in enumerate(qs):
            for r in range(rows):
                k = _keys(cache, layer, r)
                want[layer][r, :, :ctx[r]] *= decay
                want[layer][r, :, ctx[r]:len(k)] = 0
                for i, node in enumerate(paths[r]):
                    n = ctx[r] + i + 1
                    x = torch.einsum("hgd,khd->hgk", q[int(qsl[r]) + node].double().view(HKV, -1, 64), k[:n]) * 0.125
                    want[layer][r, :, :n] += x.softmax(-1).sum(1)

    qs, qsl = _step(cache, gen, [0] * rows, lens, chains)
    cache.observe(qsl)
    add(qs, qsl, [0] * rows, [range(n) for n in lens], 1.0)
    cache.held_lens.copy_(cache.seq_lens)
    parents, tokens = _trees(rows, 2, 5)
    qs, qsl = _step(cache, gen, lens, [NODES] * rows, parents)
    path, path_len, _, _ = cache.verify(torch.randn(rows * NODES, 5, generator=gen, device="cuda"),
                                        tokens.int().flatten().cuda(), torch.tensor(parents).int().flatten().cuda(), qsl,
                                        NODES, torch.full((rows,), 1.0, device="cuda"),
                                        uniforms=torch.zeros(rows * NODES, device="cuda"))  # every first child
    paths = [p[:n] for p, n in zip(path.tolist(), path_len.tolist())]
    cache.keep(qsl, path, path_len, decay=0.5)
    cache.check()
    assert cache.seq_lens.tolist() == [c + len(p) for c, p in zip(lens, paths)] and max(map(len, paths)) > 1
    add(qs, qsl, lens, paths, 0.5)
    for layer in range(2):
        for r in range(rows):
            n = int(cache.seq_lens[r])
            got, w = cache.key_weights[layer, r, :, :n].double(), want[layer][r, :, :n]
            assert torch.all((got - w).abs() <= 1.3e-4 * w + 1e-9)


@gpu
def test_eviction_keeps_what_attention_then_sees():
    """Attention over a cut cache is attention over the kept keys; pages behind it return, and rows grow on."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    rows, lens = 4, [100, 64, 65, 200]
    cache = _cache(rows)
    qs, qsl = _step(cache, gen, [0] * rows, lens, [list(range(-1, n - 1)) for n in lens])
    cache.observe(qsl)
    before = [[_keys(cache, layer, r) for r in range(rows)] for layer in range(2)]
    w = cache.key_weights.double().cpu().numpy()
    free = int(cache.free_count)
    cache.evict(64, keep_first=3, keep_last=10)
    cache.check()
    assert cache.seq_lens.tolist() == [64] * 4 and cache.evicted.tolist() == [36, 0, 1, 136]
    assert int(cache.free_count) == free + (7 - 4) + 0 + (5 - 4) + (13 - 4)
    from test_evict import kept_slots

    for layer in range(2):
        for r in range(rows):
            now = _keys(cache, layer, r)
            for h in range(HKV):
                src = kept_slots(w[layer, r, h], lens[r], 64, 3, 10) if lens[r] > 64 else np.arange(64)
                assert torch.equal(now[:, h], before[layer][r][torch.from_numpy(src).cuda(), h])
                assert np.array_equal(cache.key_weights[layer, r, h, :64].double().cpu().numpy(), w[layer, r, h, src])
    parents, _ = _trees(rows, 4, 5)
    qs, qsl = _step(cache, gen, [64] * rows, [NODES] * rows, parents)
    from _tree import ancestors

    for layer, q in enumerate(qs):
        k = cache.asked[layer][1]  # log-sum-exps
        for r in range(rows):
            keys = _keys(cache, layer, r)
            sees = torch.from_numpy(ancestors(np.array(parents[r]))[0]).cuda()
            x = torch.einsum("nhgd,khd->nhgk", q[r * NODES:(r + 1) * NODES].double().view(NODES, HKV, -1, 64), keys) * 0.125
            x[..., 64:] = x[..., 64:].masked_fill(~sees[:, None, None], -torch.inf)
            assert torch.all((x.logsumexp(-1).flatten(1) - k[r * NODES:(r + 1) * NODES]).abs() <= 1e-4)
    path = torch.zeros(rows, 1, dtype=torch.int32, device="cuda")
    cache.keep(qsl, path, torch.ones(rows, dtype=torch.int32, device="cuda"))
    cache.drop(torch.arange(rows, device="cuda"))
    cache.check()
    assert int(cache.free_count) == cache.page_refs.shape[0] and not cache.evicted.any()


@gpu
def test_forked_rows_are_refused_until_alone():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    cache = _cache(2)
    _, qsl = _step(cache, gen, [0, 0], [100, 0], [list(range(-1, 99)), []])
    cache.observe(qsl)
    cache.fork(torch.tensor([0], dtype=torch.int32, device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda"))
    assert torch.equal(cache.key_weights[:, 0], cache.key_weights[:, 1])
    cache.evict(64)
    with pytest.raises(Exception, match="UNSUPPORTED_ROW"):
        cache.check()
    assert cache.seq_lens.tolist() == [100, 100] and cache.evicted.tolist() == [0, 0]
    cache.status.zero_()
    cache.drop(torch.tensor([1], device="cuda"))
    cache.evict(64)
    cache.check()
    assert cache.seq_lens.tolist() == [64, 0]


@gpu
def test_a_budget_that_is_not_reached_changes_nothing():
    from paper_2608_22167_gb300.tree_decode import PagedCache, ToyModel, generate

    model = ToyModel(seed=2)
    plain = PagedCache(2, 3, 24, 300, model.hq, model.hkv)
    counted = PagedCache(2, 3, 24, 300, model.hq, model.hkv, count_weights=True)
    for heat in (0.0, 0.9):
        a = generate(model, plain, [1, 2, 3], 6, seed=4, nodes=10, temperature=heat)
        b = generate(model, counted, [1, 2, 3], 6, seed=4, nodes=10, temperature=heat, budget=300)
        assert a == b and torch.equal(plain.seq_lens, counted.seq_lens)
    assert not counted.evicted.any()


@gpu
def test_generation_in_a_budget_runs_on():
    from paper_2608_22167_gb300.tree_decode import PagedCache, ToyModel, generate

    model = ToyModel(seed=3)
    cache = PagedCache(2, 4, 24, 300, model.hq, model.hkv, count_weights=True)
    made = generate(model, cache, [0, 1, 2, 3], 40, seed=6, nodes=10, temperature=0.8, budget=40, keep_first=2, keep_last=8)
    lens = torch.tensor([len(x) for x in made], device="cuda")
    assert torch.equal(cache.seq_lens + cache.evicted, lens.int())  # all but the last token, and the first
    assert int(cache.seq_lens.max()) <= 40 and int(cache.evicted.max()) > 0


@gpu
def test_a_captured_round_follows_its_inputs():
    """extend, append, attend, verify, keep, weights, evict and release as one graph, against the same calls one by one."""
    from paper_2608_22167_gb300.tree_decode import rope_table, tree_masks

    rows, vocab = 3, 40
    ones, tab = torch.ones(64, device="cuda"), rope_table(2000)
    qsl = torch.arange(0, rows * NODES + 1, NODES, dtype=torch.int32, device="cuda")
    rounds = []
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    for seed in range(6):
        parents, tokens = _trees(rows, seed, 6)
        mask, depth = tree_masks(parents)
        rounds.append(dict(
            mask=mask.cuda(), depth=depth.cuda(), parents=torch.tensor(parents).int().flatten().cuda(),
            tokens=tokens.int().flatten().cuda(), u=torch.rand(rows * NODES, generator=g, device="cuda"),
            noise=torch.empty(rows, vocab, device="cuda").exponential_(generator=g).clamp_(min=1e-30),
            logits=torch.randn(rows * NODES, vocab, generator=g, device="cuda") + 3 * (torch.arange(vocab, device="cuda") < 6),
            x=torch.randn(2, rows * NODES, HQ + 2 * HKV, 64, generator=g, device="cuda", dtype=torch.bfloat16)))
    heat = torch.tensor([0.0, 1.0, 0.7], device="cuda")

    def play(cache, t, out):
        ctx = cache.seq_lens.clone()
        pos = ((ctx + cache.evicted).repeat_interleave(NODES, output_size=rows * NODES) + t["depth"]).int()
        cache.extend(ctx + NODES)
        for layer in range(2):
            x = t["x"][layer]
            q = cache.append(layer, x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], ones, ones, 1e-6, tab, qsl, pos)
            cache.attend(layer, q, qsl, t["mask"], pos)
        path, n, token, logp = cache.verify(t["logits"], t["tokens"], t["parents"], qsl, NODES, heat, uniforms=t["u"],
                                            exponentials=t["noise"])
        cache.keep(qsl, path, n, decay=0.9)
        cache.evict(5, keep_first=1, keep_last=2, limit=7)
        for o, v in zip(out, (path, n, token, logp)):
            o.copy_(v)

    def outputs():
        i32 = dict(dtype=torch.int32, device="cuda")
        return torch.empty(rows, NODES, **i32), torch.empty(rows, **i32), torch.empty(rows, **i32), torch.empty(rows, NODES, device="cuda")

    eager, replayed = _cache(rows), _cache(rows)
    held = {k: v.clone() for k, v in rounds[0].items()}
    out, got = outputs(), outputs()
    graph = torch.cuda.CUDAGraph()
    play(_cache(rows), rounds[0], outputs())
    with torch.cuda.graph(graph):
        play(replayed, held, got)
    for t in rounds:
        play(eager, t, out)
        for k, v in t.items():
            held[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, got):
            assert torch.equal(a, b)
        assert torch.equal(eager.seq_lens, replayed.seq_lens) and torch.equal(eager.evicted, replayed.evicted)
        for r in range(rows):
            n = int(eager.seq_lens[r])
            assert torch.equal(eager.key_weights[:, r, :, :n], replayed.key_weights[:, r, :, :n])
            for layer in range(2):
                assert torch.equal(_keys(eager, layer, r), _keys(replayed, layer, r))
        want = reference(dict(logits=t["logits"].double().cpu().numpy(), draft=None, tokens=t["tokens"].cpu().numpy(),
                              parents=t["parents"].cpu().numpy(), qsl=qsl.cpu().numpy(), heat=heat.cpu().numpy(),
                              u=t["u"].cpu().numpy(), noise=t["noise"].cpu().numpy(), most=NODES))
        assert want[4] > 1e-4
        for a, b in zip(out[:3], want[:3]):
            assert np.array_equal(a.cpu().numpy(), b)
    eager.check()
    replayed.check()
    assert int(eager.evicted.sum()) > 0


def test_windowed_caches_count_no_weights():
    with pytest.raises(ValueError):
        _cache(1, device="cpu", sliding_window=64)


@gpu
def test_layers_with_windows_of_their_own():
    """Each layer's weights are those of its attention: a query's sum to one, and keys before its window get none (a
    term is good to 2.2e-5, and 1e-4 of the log-sum-exp)."""
    from paper_2608_22167_gb300.tree_decode import rope_table, tree_masks

    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    rows, lens, windows = 2, [70, 31], [0, 20, 128]
    cache = _cache(rows, layers=3)
    chains = [list(range(-1, n - 1)) for n in lens]
    qsl = torch.tensor([0, 70, 101], dtype=torch.int32, device="cuda")
    cache.extend(torch.tensor(lens, device="cuda"))
    ones, tab = torch.ones(64, device="cuda"), rope_table(200)
    qs = []
    for layer, window in enumerate(windows):
        mask, depth = tree_masks(chains, window)
        x = torch.randn(sum(lens), HQ + 2 * HKV, 64, generator=gen, device="cuda", dtype=torch.bfloat16)
        q = cache.append(layer, x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], ones, ones, 1e-6, tab, qsl, depth.cuda())
        cache.attend(layer, q, qsl, mask.cuda(), depth.cuda(), sliding_window=window)
        qs.append(q)
    cache.observe(qsl)
    cache.check()
    for layer, window in enumerate(windows):
        for r, n in enumerate(lens):
            k, q = _keys(cache, layer, r), qs[layer][int(qsl[r]):int(qsl[r + 1])].double().view(n, HKV, -1, 64)
            x = torch.einsum("nhgd,khd->nhgk", q, k) * 0.125
            ahead = torch.arange(n, device="cuda")[:, None] - torch.arange(n, device="cuda")
            hidden = (ahead < 0) | (ahead >= (window or n))
            want = x.masked_fill(hidden[:, None, None], -torch.inf).softmax(-1).sum((0, 2))
            got = cache.key_weights[layer, r, :, :n].double()
            assert torch.all((got - want).abs() <= 1.3e-4 * want + 1e-9)


def test_buffers_that_layers_share_are_refused():
    """A counting cache holds each layer's q and log-sum-exps until they are counted."""
    cache = _cache(1, device="cpu")
    q, lse = torch.zeros(3, 4, HQ, 64, dtype=torch.bfloat16), torch.zeros(3, 4, HQ)
    cache._hold(0, q[0], lse[0], 0.125, 0)
    qsl, mask = torch.zeros(2, dtype=torch.int32), torch.zeros(4, 1, dtype=torch.int32)
    for bad in (dict(q=q[0], lse=lse[1]), dict(q=q[1], lse=lse[0]), dict(q=q.view(12, HQ, 64)[3:7]),
                dict(q=q[1], lse=lse.view(12, HQ)[3:7]), dict(q=q[1], out=q[0]), dict(q=q[1], out=q[1])):
        with pytest.raises(ValueError, match="counted"):
            cache.attend(1, bad.pop("q"), qsl, mask, **bad)
    kv, ones = torch.zeros(4, HKV, 64, dtype=torch.bfloat16), torch.ones(64)
    with pytest.raises(ValueError, match="counted"):
        cache.append(1, q[2], kv, kv, ones, ones, 1e-6, torch.zeros(9, 64), qsl, q_out=q[0])
    assert cache.asked[1] is None
    # other buffers, and the layer's own, get as far as the kernels' own checks
    for good in (dict(layer=1, q=q[1], lse=lse[1]), dict(layer=0, q=q[0], lse=lse[0])):
        with pytest.raises(ValueError, match="^(?!.*counted)"):
            cache.attend(good["layer"], good["q"], qsl, mask.double(), lse=good["lse"])


@gpu
@pytest.mark.parametrize("counting", [False, True])
def test_forks_of_rows_that_do_not_exist_change_no_other_row(counting):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(13)
    i32 = dict(dtype=torch.int32, device="cuda")
    if counting:
        cache = _cache(6)
    else:
        from paper_2608_22167_gb300.tree_decode import PagedCache

        cache = PagedCache(2, 6, 24, 300, HQ, HKV)
    lens = [80, 37, 0, 0, 0, 50]
    _, qsl = _step(cache, gen, [0] * 6, lens, [list(range(-1, n - 1)) for n in lens])
    if counting:
        cache.observe(qsl)
        cache.evict(48, keep_first=2, keep_last=5)
        assert cache.evicted.tolist() == [32, 0, 0, 0, 0, 2]
    cache.check()
    before = (cache.seq_lens.tolist(), cache.evicted.tolist(), None if not counting else cache.key_weights.clone())
    for src, dst in (([-1, 0, 9, 1, 5, 3], [3, 2, 4, 77, -1, 3]), ([-1], [1]), ([6], [0]), ([1], [6])):
        cache.fork(torch.tensor(src, **i32), torch.tensor(dst, **i32))
        assert cache.status.item() == 2
        cache.status.zero_()
    lens, evicted, weights = before
    lens[2], evicted[2] = lens[0], evicted[0]  # the one pair that names two rows
    assert cache.seq_lens.tolist() == lens and cache.evicted.tolist() == evicted
    if counting:
        weights[:, 2] = weights[:, 0]
        assert torch.equal(cache.key_weights, weights)


@gpu
def test_slots_taken_again_start_without_weights():
    """Rows that are dropped or cut leave no weights behind: where a later step is not counted, its keys have none."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(14)
    rows, lens = 3, [100, 90, 40]
    cache = _cache(rows)
    chains = [list(range(-1, n - 1)) for n in lens]
    _, qsl = _step(cache, gen, [0] * rows, lens, chains)
    cache.observe(qsl)
    cache.drop(torch.tensor([1], device="cuda"))
    cache.evict(64, keep_first=3, keep_last=10)
    cache.check()
    assert cache.seq_lens.tolist() == [64, 0, 40]
    for r, n in enumerate((64, 0, 40)):
        assert torch.all(cache.key_weights[:, r, :, :n] > 0) and not cache.key_weights[:, r, :, n:].any()
    # a prompt, and more of it, that nobody counts; then one token that is counted
    cache.held_lens.copy_(cache.seq_lens)
    before = cache.key_weights.clone()
    _step(cache, gen, [64, 0, 40], [30, 50, 2], [list(range(-1, n - 1)) for n in (30, 50, 2)])
    cache.held_lens.copy_(cache.seq_lens)
    _, qsl = _step(cache, gen, [94, 50, 42], [1, 1, 1], [[-1]] * 3)
    cache.observe(qsl)
    cache.check()
    added = cache.key_weights - before
    g = HQ // HKV
    want = torch.full((rows,), float(g), device="cuda", dtype=torch.float64)  # one query of g heads a kv head, 2.2e-5 + 1e-4
    assert torch.all((added.double().sum(3) - want[None, :, None]).abs() <= 1.3e-4 * g + 150 * 2.0 ** -24 * 8)


def test_steps_that_cannot_be_counted_are_refused():
    from paper_2608_22167_gb300.tree_decode import PagedCache

    cache, plain = _cache(1, device="cpu"), PagedCache(2, 1, 24, 300, HQ, HKV, device="cpu")
    qsl, path, n = (torch.zeros(s, dtype=torch.int32) for s in ((2,), (1, 1), (1,)))
    lens = cache.seq_lens.clone()
    for held in ([None, None], [(None, None, 0.125, 0), None]):  # nothing attended, or one layer of two
        cache.asked = list(held)
        for call in (lambda: cache.observe(qsl), lambda: cache.keep(qsl, path, n)):
            with pytest.raises(ValueError, match="attended"):
                call()
        assert cache.asked == held and torch.equal(cache.seq_lens, lens)
    for call in (lambda: plain.evict(64), lambda: plain.observe(qsl)):
        with pytest.raises(ValueError, match="count_weights"):
            call()


@gpu
def test_what_was_held_is_let_go_where_it_no_longer_fits():
    """Lengths or slots that changed since the attention would give its weights to other keys."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(12)
    cache = _cache(1)
    for change in (lambda: cache.extend(cache.seq_lens + 1), lambda: cache.evict(40)):
        _, qsl = _step(cache, gen, cache.seq_lens.tolist(), [20], [list(range(-1, 19))])
        change()
        with pytest.raises(ValueError, match="attended"):
            cache.observe(qsl)
    cache.check()
