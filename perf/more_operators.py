"""Measured cases of the end of a drafted round: which tokens stay, which keys mattered, which keys stay.

``verify`` walks down each row's drafted tree against the target model's
probabilities, from given random numbers, and returns the accepted path, the
next token and the log-probabilities of what was emitted. ``weights`` adds, for
every cached key, the attention weight that the step's queries gave it.
``evict`` cuts rows that have grown past a limit down to a budget of keys per kv
head: the first ones, the last ones and those of the highest weight.

``own`` False computes each pass in plain torch operations; ``own`` True makes
the calls of ``paper_2608_22167_gb300.mcpu``.
"""
import math

import numpy as np
import torch

own = False

PAGE, DIM = 16, 64
DEV = "cuda"
PEAKS = 4  # tokens of a node that stand out of its distribution


# ------------------------------------------------------------------- cases
def listed():
    return [
        # two rows with small trees and a small vocabulary: the latency of a verification
        dict(name="verify_tiny", kind="verify", rows=2, len_lo=3, len_hi=8, vocab=32000, fp32=False, greedy=False,
             draft=False, chain=False),
        # greedy decoding of 64 rows with trees of 4 to 28 nodes
        dict(name="verify_greedy", kind="verify", rows=64, len_lo=4, len_hi=28, vocab=131072, fp32=False, greedy=True,
             draft=False, chain=False),
        # the same sampled, children being the draft's likeliest tokens; rows of logits that start at odd addresses
        dict(name="verify_sampled", kind="verify", rows=64, len_lo=4, len_hi=28, vocab=100003, fp32=False,
             greedy=False, draft=False, chain=False),
        # sampled drafts with the distributions they were drawn from, chains of 2 to 8
        dict(name="verify_draft", kind="verify", rows=64, len_lo=2, len_hi=8, vocab=131072, fp32=False, greedy=False,
             draft=True, chain=True),
        # the rollout batch's 384 rows, chains of 1 (no draft at all) to 6, logits in 32 bits
        dict(name="verify_rollout", kind="verify", rows=384, len_lo=1, len_hi=6, vocab=131072, fp32=True,
             greedy=False, draft=False, chain=True),
        # one token of the tiny configuration's rows (8 q / 2 kv heads): latency
        dict(name="weights_tiny", kind="weights", rows=4, ctx_lo=16, ctx_hi=299, len_lo=1, len_hi=1, hq=8, hkv=2,
             window=0, decay=1.0, path=False),
        # a decode step over the decode batch's lengths (bound by reading the keys)
        dict(name="weights_decode", kind="weights", rows=64, ctx_lo=2047, ctx_hi=16383, len_lo=1, len_hi=1, hq=64,
             hkv=8, window=0, decay=1.0, path=False),
        # accepted paths of 1 to 8 nodes out of trees of up to 28, older weights fading
        dict(name="weights_path", kind="weights", rows=256, ctx_lo=1024, ctx_hi=8192, len_lo=8, len_hi=28, hq=64,
             hkv=8, window=0, decay=0.98, path=True),
        # 16 rows taking in tool observations of 64 to 2048 tokens: the largest products
        dict(name="weights_chunk", kind="weights", rows=16, ctx_lo=4096, ctx_hi=32768, len_lo=64, len_hi=2048, hq=64,
             hkv=8, window=0, decay=1.0, path=False),
        # rows that have passed a budget of 2048 keys by up to 80, one layer: latency
        dict(name="evict_step", kind="evict", rows=64, ctx_lo=2032, ctx_hi=2128, budget=2048, first=4, last=128, hkv=8,
             layers=1),
        # long prompts cut down after their prefill, one layer
        dict(name="evict_prefill", kind="evict", rows=32, ctx_lo=8192, ctx_hi=32768, budget=4096, first=16, last=512,
             hkv=8, layers=1),
        # twelve layers in one call, rows past their budget by 64 to 512
        dict(name="evict_model", kind="evict", rows=64, ctx_lo=2112, ctx_hi=2560, budget=2048, first=4, last=128,
             hkv=8, layers=12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["verify", "verify", "weights", "weights", "evict"])
    if kind == "verify":
        rows = _log_int(rng, 1, 384)
        hi = _log_int(rng, 1, 32)
        fp32, draft = rng.random() < 0.3, rng.random() < 0.4
        vocab = _log_int(rng, 500, 200000)
        # at most the logits of the largest listed case
        vocab = max(500, min(vocab, 384 * 6 * 131072 // (rows * hi * (2 if draft else 1) * (2 if fp32 else 1))))
        return dict(kind=kind, rows=rows, len_lo=rng.randint(1, hi), len_hi=hi, vocab=vocab, fp32=fp32,
                    greedy=rng.random() < 0.25, draft=draft, chain=rng.random() < 0.4)
    if kind == "weights":
        hq, hkv = rng.choice([(64, 8), (64, 8), (32, 8), (16, 8), (8, 8), (16, 2), (8, 2)])
        rows = _log_int(rng, 1, 384)
        path = rng.random() < 0.4
        hi = _log_int(rng, 1, 32 if path else min(2048, max(1, 16000 // rows)))
        # at most the pairs of (query head, key) of the largest listed case, and the keys of the decode batch
        most = min(65536, 1000000 // rows, 64 * 16 * 1000 * 18000 // (rows * hq * hi))
        ctx = _log_int(rng, 16, max(17, most))
        return dict(kind=kind, rows=rows, ctx_lo=rng.randint(0, ctx), ctx_hi=ctx, len_lo=rng.randint(1, hi),
                    len_hi=hi, hq=hq, hkv=hkv, window=rng.choice([0, 0, 0, 128, 37]),
                    decay=rng.choice([1.0, 1.0, 0.0, 0.9, 0.99]), path=path)
    budget = _log_int(rng, 32, 4096)
    first, last = rng.randint(0, budget // 8), rng.randint(0, budget // 4)
    layers = rng.randint(1, 12)
    rows = _log_int(rng, 1, 128)
    hi = max(budget + 1, min(_log_int(rng, budget + 1, 16 * budget), 64 * 12 * 2336 // (rows * layers)))
    return dict(kind=kind, rows=rows, ctx_lo=rng.randint(budget // 2, hi), ctx_hi=hi, budget=budget, first=first,
                last=last, hkv=rng.choice([8, 8, 4, 2, 1]), layers=layers)


# ------------------------------------------------------------------ inputs
def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly spread: the same for every seed."""
    return np.rint(np.linspace(lo, hi, n)).astype(np.int64) if n > 1 else np.array([(lo + hi) // 2], np.int64)


def _put(x, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=dtype, device=DEV)


def _starts(lens):
    return np.concatenate([[0], np.cumsum(lens)])


def _tables(total, longest, rng, pages):
    """A scattered block table in a pool of `pages` for rows of `total` tokens, `longest` at most."""
    last = -(-total // PAGE)
    need = np.arange(-(-longest // PAGE))[None, :] < last[:, None]
    table = np.full(need.shape, -1, np.int32)
    table[need] = rng.permutation(pages)[: int(need.sum())]
    return table


def _trees(lens, rng, chain):
    """Parents (-1: the first node) of one random tree a row, nodes in topological order, and the nodes' ranks among
    their siblings."""
    parents, ranks = [], []
    for n in lens:
        born = [0] * int(n)
        for i in range(int(n)):
            up = i - 1 if chain or i == 0 else i - min(int(rng.integers(1, 5)), i)
            parents.append(up)
            ranks.append(born[up] if up >= 0 else 0)
            if up >= 0:
                born[up] += 1
    return np.array(parents), np.array(ranks)


def prepare(case, seed):
    rng = np.random.default_rng([seed, 21])
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return dict(verify=_prepare_verify, weights=_prepare_weights, evict=_prepare_evict)[case["kind"]](case, rng, gen)


def _prepare_verify(case, rng, gen):
    rows, vocab = case["rows"], case["vocab"]
    lens = rng.permutation(_spread(case["len_lo"], case["len_hi"], rows))
    total = int(lens.sum())
    parents, ranks = _trees(lens, rng, case["chain"])
    starts = _starts(lens)
    up = np.maximum(parents, 0) + np.repeat(starts[:-1], lens)  # the parent's query token
    dtype = torch.float32 if case["fp32"] else torch.bfloat16
    logits = torch.empty(total, vocab, dtype=dtype, device=DEV)
    draft = torch.empty(total, vocab, dtype=dtype, device=DEV) if case["draft"] else None
    stand = _put(rng.integers(0, vocab, size=(total, PEAKS)), torch.int64)
    height = math.log(vocab) + 4.5 - torch.arange(PEAKS, device=DEV)
    width = int(ranks.max()) + 1
    drawn = torch.empty(total, width, dtype=torch.int64, device=DEV)  # tokens drawn from the draft at each node
    step = max(1, (1 << 27) // vocab)
    for a in range(0, total, step):
        b = min(total, a + step)
        x = 2 * torch.randn(b - a, vocab, generator=gen, device=DEV)
        x.scatter_(1, stand[a:b], height + 0.3 * torch.randn(b - a, PEAKS, generator=gen, device=DEV))
        logits[a:b] = x
        if case["draft"]:
            draft[a:b] = x + 0.7 * torch.randn(b - a, vocab, generator=gen, device=DEV)
            drawn[a:b] = torch.multinomial(draft[a:b].float().div(0.8).softmax(1), width, True, generator=gen)
    parent_t, rank_t = _put(up, torch.int64), _put(ranks, torch.int64)
    if case["draft"]:
        tokens = drawn[parent_t, rank_t]
    else:
        tokens = stand[parent_t, rank_t.clamp(max=PEAKS - 1)]
        stray = (torch.rand(total, generator=gen, device=DEV) < 0.15) | (rank_t >= PEAKS)
        tokens = torch.where(stray, torch.randint(0, vocab, (total,), generator=gen, device=DEV), tokens)
    depth = np.zeros(total, np.int64)
    for i in range(total):
        depth[i] = depth[up[i]] + 1 if parents[i] >= 0 else 0
    deep, most = int(depth.max()) + 1, case["len_hi"]
    i32 = dict(dtype=torch.int32, device=DEV)
    return dict(case=case, kind="verify", rows=rows, lens=lens.tolist(), width=width, deep=deep, most=most, logits=logits,
                draft=draft, tokens=tokens.int(), parents=_put(parents), qsl=_put(starts),
                temperature=torch.full((rows,), 0.0 if case["greedy"] else 0.8, device=DEV),
                uniforms=torch.rand(total, generator=gen, device=DEV),
                exponentials=torch.empty(rows, vocab, device=DEV).exponential_(generator=gen).clamp_(min=1e-9),
                path=torch.empty(rows, most, **i32), path_len=torch.empty(rows, **i32),
                next=torch.empty(rows, **i32), logprobs=torch.empty(rows, most, device=DEV),
                status=torch.zeros(1, **i32))


def _prepare_weights(case, rng, gen):
    rows, hq, hkv = case["rows"], case["hq"], case["hkv"]
    ctx = rng.permutation(_spread(case["ctx_lo"], case["ctx_hi"], rows))
    lens = rng.permutation(_spread(case["len_lo"], case["len_hi"], rows))
    taken, path, path_len = lens, None, None
    if case["path"]:
        # the accepted nodes, moved behind the context: their queries are some of the tree's
        taken = np.minimum(lens, 1 + rng.permutation(np.arange(rows) % 8))
        path = np.zeros((rows, int(taken.max())), np.int64)
        for r in range(rows):
            path[r, : taken[r]] = np.sort(np.r_[0, 1 + rng.permutation(int(lens[r]) - 1)[: taken[r] - 1]])
        path_len = taken
    total = ctx + taken
    # room for any order of the lengths, so that the pool has one size for all seeds
    most = min(int(lens.max()), 8) if case["path"] else None
    pages = int((-(-ctx // PAGE)).sum() + (rows * -(-most // PAGE) if most else (-(-lens // PAGE)).sum())) + 1
    table = _tables(total, int(ctx.max() + lens.max()), rng, pages)
    t = int(lens.sum())

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)

    # log-sum-exps of normal scores over the keys that a query sees
    seen = np.repeat(total, lens).astype(np.float64)
    if case["window"] > 0:
        seen = np.minimum(seen, case["window"])
    lse = _put(np.log(seen) + 0.5, torch.float32)[:, None] + 0.1 * torch.randn(t, hq, generator=gen, device=DEV)
    slots = table.shape[1] * PAGE
    s = dict(case=case, kind="weights", rows=rows, ctx=ctx.tolist(), lens=lens.tolist(), taken=taken.tolist(),
             q=randn(t, hq, DIM), kc=randn(pages, hkv, PAGE, DIM), lse=lse, bt=_put(table), sl=_put(total),
             qsl=_put(_starts(lens)), starts=_starts(lens).tolist(), scale=DIM ** -0.5,
             path=None if path is None else _put(path), path_len=None if path_len is None else _put(path_len),
             weights=torch.rand(rows, hkv, slots, generator=gen, device=DEV).pow_(4).mul_(8))
    if own:
        from paper_2608_22167_gb300 import mcpu

        s["ws"] = mcpu.new_weights_workspace(mcpu.dims(s["q"], s["kc"], s["bt"], s["sl"]), DEV)
    return s


def _prepare_evict(case, rng, gen):
    rows, hkv, layers = case["rows"], case["hkv"], case["layers"]
    total = rng.permutation(_spread(case["ctx_lo"], case["ctx_hi"], rows))
    pages = int((-(-total // PAGE)).sum()) + 1
    table = _tables(total, int(total.max()), rng, pages)
    slots = table.shape[1] * PAGE
    pools = torch.randn(2 * layers, pages, hkv, PAGE, DIM, generator=gen, device=DEV, dtype=torch.bfloat16)
    # few keys get most of the attention, many next to none; some have exactly the same
    w = torch.randn(layers, rows, hkv, slots, generator=gen, device=DEV).mul_(2).exp_()
    w = torch.where(w < 0.05, torch.zeros((), device=DEV), w)
    s = dict(case=case, kind="evict", rows=rows, total=total.tolist(), pools=pools, bt=_put(table), sl=_put(total),
             weights=w, new_weights=torch.zeros_like(w), refs=torch.zeros(pages, dtype=torch.int32, device=DEV),
             new_lens=torch.empty(rows, dtype=torch.int32, device=DEV),
             status=torch.zeros(1, dtype=torch.int32, device=DEV))
    if own:
        from paper_2608_22167_gb300 import mcpu

        s["list"] = mcpu.PoolList(list(pools))
    return s


# -------------------------------------------------------------------- work
def _lengths(case):
    n = case["rows"]
    return _spread(case["ctx_lo"], case["ctx_hi"], n)


def work(case):
    if case["kind"] == "verify":
        # a walk visits 2 to 3 nodes where it can (about three drafted tokens in five are accepted), and reads a row of
        # exponentials once it samples
        lens = _spread(case["len_lo"], case["len_hi"], case["rows"])
        visits = sum(sum(0.6 ** d for d in range(min(int(n), 5))) for n in lens)
        logits = visits * (2 if case["draft"] and not case["greedy"] else 1)
        size = 4 if case["fp32"] else 2
        return dict(bytes=case["vocab"] * (logits * size + (0 if case["greedy"] else 4 * case["rows"])),
                    flops=4.0 * case["vocab"] * logits)
    ctx = _lengths(case)
    if case["kind"] == "weights":
        hq, hkv, w = case["hq"], case["hkv"], case["window"]
        lens = _spread(case["len_lo"], case["len_hi"], case["rows"])
        taken = np.minimum(lens, 4) if case["path"] else lens
        # the lengths come in any order: sums of products by the means
        mean, n = float(ctx.mean()), case["rows"]
        keys = np.minimum(ctx, w) + taken if w > 0 else ctx + taken
        pairs = sum(min(mean, w) * float(t) if w > 0 else mean * float(t) + float(t) * (float(t) + 1) / 2 for t in taken)
        # old weights are read and written wherever they change
        old = keys.sum() if case["decay"] == 1.0 else (ctx + taken).sum()
        return dict(bytes=float(keys.sum() * hkv * DIM * 2 + old * hkv * (4 if case["decay"] == 0 else 8)
                                + taken.sum() * hq * (DIM * 2 + 4)), flops=2.0 * DIM * hq * pairs)
    first, last, budget = case["first"], case["last"], case["budget"]
    read = moved = kept = 0.0
    for n in ctx:
        n = int(n)
        read += n
        kept += min(n, budget)
        if n > budget:
            # of the keys past the new end as many are kept as of all that are not the first or the last
            moved += (n - budget) * (budget - first - last) / max(1, n - first - last) + last
    heads = case["hkv"] * case["layers"]
    return dict(bytes=heads * (4 * read + 4 * kept + moved * 2 * 2 * DIM * 2), flops=float(heads * read))


# --------------------------------------------------------------------- run
def run(state):
    return dict(verify=_verify, weights=_weights, evict=_evict)[state["kind"]](state)


def _verify(s):
    if own:
        from paper_2608_22167_gb300 import mcpu

        mcpu.mcpu_verify_tree(s["logits"], s["tokens"], s["parents"], s["qsl"], s["temperature"], s["uniforms"],
                              s["exponentials"], s["path"], s["path_len"], s["next"], s["logprobs"], s["status"],
                              draft_logits=s["draft"])
        return dict(path=s["path"], path_len=s["path_len"], next=s["next"], logprobs=s["logprobs"])
    greedy, rows, most, deep, width = s["case"]["greedy"], s["rows"], s["most"], s["deep"], s["width"]
    first, total = s["qsl"][:-1].long(), s["tokens"].shape[0]
    every = torch.arange(rows, device=DEV)
    # children of every node, in ascending order: node numbers in the batch, `total` for none
    node = torch.arange(total, device=DEV)
    row = torch.searchsorted(s["qsl"].long(), node, right=True) - 1
    up = torch.where(s["parents"] < 0, total, first[row] + s["parents"])
    order = torch.argsort(up, stable=True)
    rank = torch.arange(total, device=DEV) - torch.searchsorted(up[order], up[order])
    children = torch.full((total + 1, max(width, 1)), total, device=DEV)
    children[up[order], rank.clamp(max=width - 1)] = order
    children = torch.cat([children[:total], torch.full((1, max(width, 1)), total, device=DEV)])
    tokens = torch.cat([s["tokens"].long(), torch.zeros(1, dtype=torch.int64, device=DEV)])
    uniforms = torch.cat([s["uniforms"].double(), torch.ones(1, dtype=torch.float64, device=DEV)])
    heat = 1.0 if greedy else s["temperature"].double()[:, None]
    path = torch.full((rows, most), -1, dtype=torch.int64, device=DEV)
    logprobs = torch.zeros(rows, most, dtype=torch.float64, device=DEV)
    done = torch.zeros(rows, dtype=torch.bool, device=DEV)
    path[:, 0] = 0
    length, following, cur = torch.ones_like(first), torch.full_like(first, -1), first.clone()
    for level in range(deep):
        # 64 bits: a draw next to a border, and long sums
        logp = torch.log_softmax(s["logits"][cur].double() / heat, 1)
        p = logp.exp()
        taken = torch.full_like(cur, total)
        best = s["logits"][cur].float().argmax(1) if greedy else None
        q = torch.softmax(s["draft"][cur].double() / heat, 1) if s["draft"] is not None and not greedy else None
        rest, mass, gone = p, torch.ones(rows, 1, dtype=torch.float64, device=DEV), 0.0
        for c in range(width if level + 1 < deep else 0):
            kid = children[cur, c]
            x = tokens[kid][:, None]
            live = (kid < total) & (taken == total)
            if greedy:
                ok = live & (x[:, 0] == best)
            elif q is None:
                ok = live & ((uniforms[kid][:, None] * mass) < rest.gather(1, x))[:, 0]
            else:
                ok = live & ((uniforms[kid][:, None] * mass * q.gather(1, x)) < rest.gather(1, x))[:, 0]
            taken = torch.where(ok, kid, taken)
            lost = (live & ~ok)[:, None]
            if not greedy:
                if q is None:
                    less = rest.scatter(1, x, 0.0)
                else:
                    gone = gone + torch.where(lost, mass, 0.0)
                    less = (p - gone * q).clamp(min=0)
                rest = torch.where(lost, less, rest)
                mass = torch.where(lost, less.sum(1, keepdim=True), mass)
        if greedy:
            pick = best
        else:
            rest = torch.where(rest.amax(1, keepdim=True) > 0, rest, p)
            pick = (rest / s["exponentials"].double()).argmax(1)
        go = taken < total
        out = torch.where(go, tokens[taken], pick)
        # the row's walk ends where no child was accepted
        logprobs[:, level] = torch.where(done, 0.0, logp[every, out])
        following = torch.where(done | go, following, pick)
        done = done | ~go
        if level + 1 < deep:
            path[:, level + 1] = torch.where(done, -1, taken - first)
            length = length + (~done).long()
        cur = torch.where(done, cur, taken)
    return dict(path=path.int(), path_len=length.int(), next=following.int(), logprobs=logprobs.float())


def _slots(s, r, n):
    """Physical page and slot of positions 0 .. n - 1 of row r."""
    at = torch.arange(n, device=DEV)
    return s["bt"][r, at // PAGE].long(), at % PAGE


def _weights(s):
    case = s["case"]
    if own:
        from paper_2608_22167_gb300 import mcpu

        mcpu.mcpu_accumulate_weights(s["q"], s["lse"], s["kc"], s["bt"], s["sl"], s["qsl"], case["window"], s["scale"],
                                     case["decay"], s["weights"], s["ws"], query_path=s["path"],
                                     path_len=s["path_len"])
        return dict(weights=s["weights"])
    hkv, group = case["hkv"], case["hq"] // case["hkv"]
    for r in range(s["rows"]):
        ctx, n, a = s["ctx"][r], s["taken"][r], s["starts"][r]
        q, lse = s["q"][a : a + s["lens"][r]], s["lse"][a : a + s["lens"][r]]
        if case["path"]:
            at = s["path"][r, :n].long()
            q, lse = q[at], lse[at]
        page, slot = _slots(s, r, ctx + n)
        k = s["kc"][page, :, slot].float()  # [keys, hkv, dim]
        pos = torch.arange(ctx + n, device=DEV)
        new = torch.zeros(hkv, ctx + n, device=DEV)
        step = max(1, (1 << 28) // ((ctx + n) * group))
        for i in range(0, n, step):
            own_pos = ctx + torch.arange(i, min(n, i + step), device=DEV)
            sees = pos[None] <= own_pos[:, None]
            if case["window"] > 0:
                sees &= own_pos[:, None] - pos[None] < case["window"]
            for h in range(hkv):
                x = q[i : i + step, h * group : (h + 1) * group].float() @ k[:, h].T * s["scale"]
                x = (x - lse[i : i + step, h * group : (h + 1) * group, None]).exp()
                new[h] += torch.where(sees[:, None], x, 0.0).sum((0, 1))
        if case["decay"] != 0:
            new[:, :ctx] += case["decay"] * s["weights"][r, :, :ctx]
        s["weights"][r, :, : ctx + n] = new
    return dict(weights=s["weights"])


def _evict(s):
    case = s["case"]
    if own:
        from paper_2608_22167_gb300 import mcpu

        mcpu.mcpu_evict_kv(s["list"], s["weights"], s["bt"], s["sl"], case["budget"], case["budget"], case["first"],
                           case["last"], s["new_weights"], s["new_lens"], s["status"], page_refs=s["refs"])
        return dict(pools=s["pools"], weights=s["new_weights"], lens=s["new_lens"])
    first, last, budget, layers, hkv = case["first"], case["last"], case["budget"], case["layers"], case["hkv"]
    for r in range(s["rows"]):
        n = s["total"][r]
        s["new_weights"][:, r, :, : min(n, budget)] = s["weights"][:, r, :, : min(n, budget)]
        if n <= budget:
            continue
        # the middle keys to keep, by weight and, among equals, by slot
        order = torch.sort(s["weights"][:, r, :, first : n - last], dim=2, descending=True, stable=True).indices
        keep = torch.zeros(layers, hkv, n, dtype=torch.bool, device=DEV)
        keep[:, :, first : n - last].scatter_(2, order[:, :, : budget - first - last], True)
        inner = budget - last
        slot = torch.arange(budget, device=DEV)
        hole = (slot[:inner] >= first) & ~keep[:, :, :inner]
        # kept keys past the new middle, in ascending order, for the holes in ascending order
        late = torch.argsort(keep[:, :, inner:].byte(), dim=2, descending=True, stable=True) + inner
        rank = (hole.cumsum(2) - 1).clamp(min=0, max=late.shape[2] - 1)
        src = torch.cat([torch.where(hole, late.gather(2, rank), slot[:inner]),
                         torch.arange(n - last, n, device=DEV).expand(layers, hkv, -1)], 2)
        layer = torch.arange(layers, device=DEV)[:, None, None]
        head = torch.arange(hkv, device=DEV)[None, :, None]
        bt = s["bt"][r].long()
        for half in range(2):
            pools = s["pools"][half * layers : (half + 1) * layers]
            pools[layer, bt[slot // PAGE], head, slot % PAGE] = pools[layer, bt[src // PAGE], head, src % PAGE]
        s["new_weights"][:, r, :, :budget] = s["weights"][:, r].gather(2, src)
    return dict(pools=s["pools"], weights=s["new_weights"], lens=s["sl"].clamp(max=budget))


# ------------------------------------------------------------------- exact
def exact(case, seed):
    s = prepare(case, seed)
    return dict(verify=_exact_verify, weights=_exact_weights, evict=_exact_evict)[case["kind"]](s)


def _exact_verify(s):
    case, qsl = s["case"], s["qsl"].tolist()
    parents, tokens, uniforms = s["parents"].tolist(), s["tokens"].tolist(), s["uniforms"].double().tolist()
    path = torch.full((s["rows"], s["most"]), -1, dtype=torch.int32)
    logprobs = torch.zeros(s["rows"], s["most"], dtype=torch.float64)
    length, following = [], []
    for r in range(s["rows"]):
        a, b = qsl[r], qsl[r + 1]
        heat = 1.0 if case["greedy"] else float(s["temperature"][r].double())
        walk = [0]
        while True:
            at = walk[-1]
            x = s["logits"][a + at].double() / heat
            logp = x - torch.logsumexp(x, 0)
            left = logp.exp()
            if case["draft"]:
                y = s["draft"][a + at].double() / heat
                q = (y - torch.logsumexp(y, 0)).exp()
            kids = [i for i in range(at + 1, b - a) if parents[a + i] == at] if len(walk) < s["most"] else []
            best = int((x == x.max()).nonzero()[0])
            went = None
            for i in kids:
                token = tokens[a + i]
                if case["greedy"]:
                    went = i if token == best else None
                else:
                    mass = float(left.sum())
                    chance = float(left[token]) / mass if mass > 0 else 0.0
                    if case["draft"]:
                        chance /= float(q[token])
                    went = i if uniforms[a + i] < chance else None
                    if went is None and case["draft"]:
                        left = torch.relu(left - mass * q)
                    elif went is None:
                        left = left.clone()
                        left[token] = 0.0
                if went is not None:
                    break
            if went is None:
                race = (left if float(left.max()) > 0 else logp.exp()) / s["exponentials"][r].double()
                pick = best if case["greedy"] else int((race == race.max()).nonzero()[0])
                logprobs[r, len(walk) - 1] = float(logp[pick])
                break
            logprobs[r, len(walk) - 1] = float(logp[tokens[a + went]])
            walk.append(went)
        path[r, : len(walk)] = torch.tensor(walk, dtype=torch.int32)
        length.append(len(walk))
        following.append(pick)
    return dict(path=path.to(DEV), path_len=torch.tensor(length, dtype=torch.int32, device=DEV),
                next=torch.tensor(following, dtype=torch.int32, device=DEV), logprobs=logprobs.to(DEV))


def _exact_weights(s):
    case = s["case"]
    group = case["hq"] // case["hkv"]
    out = s["weights"].double()
    bt = s["bt"].tolist()
    for r in range(s["rows"]):
        a, n = s["starts"][r], s["taken"][r]
        end = s["ctx"][r] + n
        rows = s["path"][r, :n].long() + a if case["path"] else torch.arange(a, a + n, device=DEV)
        k = torch.cat([s["kc"][p] for p in bt[r][: -(-end // PAGE)]], 1)[:, :end].double()  # [hkv, keys, dim]
        out[r, :, end - n : end] = 0
        out[r, :, : end - n] *= case["decay"]
        key = torch.arange(end, device=DEV)
        step = max(1, (1 << 27) // end)
        for h in range(case["hkv"]):
            for g in range(group):
                for i in range(0, n, step):
                    t = rows[i : i + step]
                    x = torch.einsum("nd,kd->nk", s["q"][t, h * group + g].double(), k[h]) * s["scale"]
                    x = torch.exp(x - s["lse"][t, h * group + g].double()[:, None])
                    ahead = (end - n + i + torch.arange(len(t), device=DEV))[:, None] - key
                    hidden = ahead < 0
                    if case["window"] > 0:
                        hidden |= ahead >= case["window"]
                    out[r, h, :end] += x.masked_fill(hidden, 0).sum(0)
    return dict(weights=out)


def _exact_evict(s):
    case = s["case"]
    first, last, budget = case["first"], case["last"], case["budget"]
    w = s["weights"].double().cpu().numpy()
    out = np.zeros_like(w)
    pools = s["pools"].double()
    bt = s["bt"].cpu().numpy().astype(np.int64)
    for r, n in enumerate(s["total"]):
        out[:, r, :, : min(n, budget)] = w[:, r, :, : min(n, budget)]
        if n <= budget:
            continue
        for m in range(case["layers"]):
            for h in range(case["hkv"]):
                v = w[m, r, h, :n]
                # middle slots by falling weight, then by rising slot
                rank = np.lexsort((np.arange(first, n - last), -v[first : n - last])) + first
                kept = np.sort(rank[: budget - first - last])
                inner = budget - last
                holes = np.setdiff1d(np.arange(first, inner), kept)
                old = np.concatenate([kept[kept >= inner], np.arange(n - last, n)])
                new = np.concatenate([holes, np.arange(inner, budget)])
                out[m, r, h, new] = v[old]
                op, np_ = torch.as_tensor(bt[r, old // PAGE], device=DEV), torch.as_tensor(bt[r, new // PAGE], device=DEV)
                os_, ns = torch.as_tensor(old % PAGE, device=DEV), torch.as_tensor(new % PAGE, device=DEV)
                for i in (m, m + case["layers"]):
                    pools[i, np_, h, ns] = pools[i, op, h, os_].clone()
    return dict(pools=pools, weights=torch.as_tensor(out, device=DEV), lens=None)
