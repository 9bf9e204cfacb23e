"""Measured cases of one round of tree-drafted decoding over the paged KV cache.

A draft model proposes a small tree of tokens for every row of the batch. The
round then normalises and rotates the queries and keys of all drafted tokens
and writes K and V into the rows' pages (``norm_rope``), lets every drafted
token attend to its row's context and to its own ancestors (``tree``), moves
the K/V rows of the accepted path to the front (``compact``), and, when a
search or a new set of samples starts, drops the previous samples' pages and
forks new rows from the prompts (``pages``: release, fork, tail-page copy).

``own`` False computes each pass in plain torch operations in 32 bits; ``own``
True makes the calls of ``paper_2608_22167_gb300.mcpu``.
"""
import math

import numpy as np
import torch

own = False

PAGE, DIM = 16, 64
DEV = "cuda"


# ------------------------------------------------------------------- cases
def listed():
    return [
        # one plain decode step of 64 rows, one layer: the latency of the call
        dict(name="norm_decode", kind="norm", rows=64, len_lo=1, len_hi=1, prior_lo=0, prior_hi=4096, hq=64, hkv=8,
             packed=True, depth=False),
        # 256 rows verifying trees of 4 to 28 tokens, positions by depth
        dict(name="norm_tree", kind="norm", rows=256, len_lo=4, len_hi=28, prior_lo=64, prior_hi=2048, hq=64, hkv=8,
             packed=True, depth=True),
        # 32 rows taking in tool observations of 64 to 2048 tokens
        dict(name="norm_chunk", kind="norm", rows=32, len_lo=64, len_hi=2048, prior_lo=0, prior_hi=1024, hq=64, hkv=8,
             packed=False, depth=False),
        # the tiny configuration's rows (8 q / 2 kv heads), trees of up to 8 tokens: latency
        dict(name="tree_tiny", kind="tree", rows=4, ctx_lo=17, ctx_hi=300, len_lo=1, len_hi=8, hq=8, hkv=2, window=0,
             sinks=False),
        # the decode batch's lengths with small trees (bound by reading the cache)
        dict(name="tree_decode", kind="tree", rows=64, ctx_lo=2048, ctx_hi=16384, len_lo=1, len_hi=16, hq=64, hkv=8,
             window=0, sinks=True),
        # the mixed batch's lengths with wide trees: the largest products
        dict(name="tree_wide", kind="tree", rows=64, ctx_lo=4096, ctx_hi=32768, len_lo=16, len_hi=32, hq=64, hkv=8,
             window=0, sinks=False),
        # two rows at the long-horizon end of the lengths, trees of 61 and 64 tokens: few rows, one long axis
        dict(name="tree_long", kind="tree", rows=2, ctx_lo=49152, ctx_hi=65536, len_lo=61, len_hi=64, hq=64, hkv=8,
             window=0, sinks=False),
        # a sliding-window layer of the rollout batch's 384 rows
        dict(name="tree_window", kind="tree", rows=384, ctx_lo=1024, ctx_hi=24576, len_lo=4, len_hi=28, hq=64, hkv=8,
             window=128, sinks=True),
        # one layer's K and V after verification: latency
        dict(name="compact_layer", kind="compact", rows=64, ctx_lo=33, ctx_hi=512, len_lo=4, len_hi=28, hkv=8,
             layers=1),
        # the twelve full-context layers of a model in one call
        dict(name="compact_model", kind="compact", rows=256, ctx_lo=33, ctx_hi=512, len_lo=8, len_hi=32, hkv=8,
             layers=12),
        # 8 samples of 8 prompts replaced, two layers
        dict(name="pages_few", kind="pages", groups=8, samples=8, ctx_lo=253, ctx_hi=2041, hkv=8, layers=2),
        # the rollout batch's 48 groups of 8 samples, twelve layers
        dict(name="pages_rollout", kind="pages", groups=48, samples=8, ctx_lo=1024, ctx_hi=4096, hkv=8, layers=12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "tree", "tree", "compact", "pages"])
    hq, hkv = rng.choice([(64, 8), (64, 8), (32, 8), (16, 8), (8, 8), (16, 2), (8, 2)])
    if kind == "norm":
        rows = _log_int(rng, 1, 256)
        hi = _log_int(rng, 1, max(1, min(2048, 32000 // rows)))
        lo = rng.randint(1, hi)
        return dict(kind=kind, rows=rows, len_lo=lo, len_hi=hi, prior_lo=rng.randint(0, 64),
                    prior_hi=_log_int(rng, 65, 4096), hq=hq, hkv=hkv, packed=rng.random() < 0.5,
                    depth=hi <= 64 and rng.random() < 0.7)
    if kind == "tree":
        window = rng.choice([0, 0, 0, 128, 37])
        rows = _log_int(rng, 1, 384)
        hi = _log_int(rng, 1, 64)
        # at most the pairs of (query head, key) that the widest listed case pads to
        most = 64 * 64 * 32 * 32768 // (rows * hq * hi)
        ctx = _log_int(rng, 16, max(17, min(65536, 1200000 // rows, most)))
        return dict(kind=kind, rows=rows, ctx_lo=rng.randint(0, ctx), ctx_hi=ctx, len_lo=rng.randint(1, hi), len_hi=hi,
                    hq=hq, hkv=hkv, window=window, sinks=rng.random() < 0.5)
    if kind == "compact":
        hi = _log_int(rng, 1, 64)
        return dict(kind=kind, rows=_log_int(rng, 1, 256), ctx_lo=rng.randint(0, 32), ctx_hi=_log_int(rng, 33, 512),
                    len_lo=rng.randint(1, hi), len_hi=hi, hkv=hkv, layers=rng.randint(1, 12))
    return dict(kind=kind, groups=_log_int(rng, 1, 48), samples=rng.randint(1, 8), ctx_lo=rng.randint(1, 512),
                ctx_hi=_log_int(rng, 513, 4096), hkv=hkv, layers=rng.randint(1, 12))


# ------------------------------------------------------------------ inputs
def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly spread: the same for every seed."""
    return np.rint(np.linspace(lo, hi, n)).astype(np.int64) if n > 1 else np.array([(lo + hi) // 2], np.int64)


def _lengths(case, rng):
    """Context length and drafted tokens of each row, in a seeded order."""
    n = case["rows"]
    lo, hi = (case["prior_lo"], case["prior_hi"]) if case["kind"] == "norm" else (case["ctx_lo"], case["ctx_hi"])
    return rng.permutation(_spread(lo, hi, n)), rng.permutation(_spread(case["len_lo"], case["len_hi"], n))


def _first_page(ctx, window):
    """First logical page that a query of the row can see."""
    return np.maximum(ctx - window + 1, 0) // PAGE if window > 0 else np.zeros_like(ctx)


def _tables(first, total, rng, pages):
    """A scattered block table in a pool of `pages` for rows of `total` tokens, without the pages before `first`."""
    last = (total + PAGE - 1) // PAGE
    width = int(max(1, last.max()))
    j = np.arange(width)[None, :]
    need = (j >= first[:, None]) & (j < last[:, None])
    table = np.full((len(total), width), -1, np.int32)
    table[need] = rng.permutation(pages)[: int(need.sum())]
    return table


def _trees(lens, rng):
    """Ancestor masks (32-bit words) and depths of one random tree a row, nodes in topological order."""
    rows, most = len(lens), int(lens.max())
    words = (most + 31) // 32
    mask = np.zeros((rows, most, words), np.uint32)
    depth = np.zeros((rows, most), np.int64)
    every = np.arange(rows)
    for i in range(most):
        back = np.minimum(rng.integers(1, 5, size=rows), i + 1)
        parent = i - back  # -1: a child of the context
        up = np.maximum(parent, 0)
        mask[:, i] = np.where(parent[:, None] >= 0, mask[every, up], 0)
        mask[:, i, i // 32] |= np.uint32(1 << (i % 32))
        depth[:, i] = np.where(parent >= 0, depth[every, up] + 1, 0)
    node = np.arange(most)[None, :] < lens[:, None]
    return mask[node].view(np.int32), depth[node]


def _put(x, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=dtype, device=DEV)


def _starts(lens):
    return np.concatenate([[0], np.cumsum(lens)])


def prepare(case, seed):
    rng = np.random.default_rng([seed, 20])
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)

    if case["kind"] == "pages":
        return _prepare_pages(case, rng, randn)
    ctx, lens = _lengths(case, rng)
    total = ctx + lens
    window = case.get("window", 0)
    # room for any order of the lengths, so that the pool has one size for all seeds
    seen = np.minimum(ctx, window + PAGE) if window > 0 else ctx
    pages = int((-(-seen // PAGE) - (-lens // PAGE)).sum()) + 1
    table = _tables(_first_page(ctx, window), total, rng, pages)
    hkv = case["hkv"]
    s = dict(case=case, kind=case["kind"], bt=_put(table), sl=_put(total), qsl=_put(_starts(lens)),
             status=torch.zeros(1, dtype=torch.int32, device=DEV), most=int(lens.max()), rows=len(lens))
    if case["kind"] == "compact":
        s["pools"] = randn(2 * case["layers"], pages, hkv, PAGE, DIM)
        # accepted paths: increasing node numbers, from none to six of them
        most = min(6, int(lens.max()))
        path = np.zeros((len(lens), most), np.int32)
        taken = np.minimum(rng.integers(0, most + 1, size=len(lens)), lens)
        for r, (n, k) in enumerate(zip(lens, taken)):
            path[r, :k] = np.sort(rng.permutation(int(n))[:k])
        s.update(path=_put(path), taken=_put(taken), new_sl=torch.zeros(len(lens), dtype=torch.int32, device=DEV))
        if own:
            from paper_2608_22167_gb300 import mcpu
            s["list"] = mcpu.PoolList([s["pools"][i] for i in range(s["pools"].shape[0])])
        return s
    s.update(kc=randn(pages, hkv, PAGE, DIM), vc=randn(pages, hkv, PAGE, DIM))
    tokens, hq = int(lens.sum()), case["hq"]
    mask, depth = _trees(lens, rng) if case["kind"] == "tree" or case["depth"] else (None, None)
    if case["kind"] == "tree":
        s.update(q=randn(tokens, hq, DIM), mask=_put(mask), scale=DIM ** -0.5, window=window,
                 positions=_put(np.repeat(ctx, lens) + depth),
                 sinks=torch.randn(hq, generator=gen, device=DEV) * 1.5 if case["sinks"] else None,
                 out=torch.empty(tokens, hq, DIM, dtype=torch.bfloat16, device=DEV),
                 lse=torch.empty(tokens, hq, dtype=torch.float32, device=DEV),
                 span=int((total - _first_page(ctx, window) * PAGE).max()))
        if own:
            from paper_2608_22167_gb300 import mcpu
            s["ws"] = mcpu.new_tree_workspace(mcpu.dims(s["q"], s["kc"], s["bt"], s["sl"]), DEV)
        return s
    # the projection's output: q, k and v side by side in one row a token, or apart
    if case["packed"]:
        qkv = randn(tokens, (hq + 2 * hkv) * DIM) * 2
        cut = qkv.split([hq * DIM, hkv * DIM, hkv * DIM], dim=1)
        q, k, v = (x.unflatten(1, (-1, DIM)) for x in cut)
    else:
        q, k, v = randn(tokens, hq, DIM) * 2, randn(tokens, hkv, DIM) * 2, randn(tokens, hkv, DIM)
    angle = torch.arange(int(total.max()), device=DEV, dtype=torch.float64)[:, None] * \
        150000.0 ** (-torch.arange(DIM // 2, device=DEV, dtype=torch.float64) * 2 / DIM)[None, :]
    s.update(q=q, k=k, v=v, wq=1 + 0.2 * torch.randn(DIM, generator=gen, device=DEV),
             wk=1 + 0.2 * torch.randn(DIM, generator=gen, device=DEV), eps=1e-6,
             positions=_put(np.repeat(ctx, lens) + depth) if depth is not None else None,
             rope=torch.cat([angle.cos(), angle.sin()], 1).float().contiguous(),
             q_out=torch.empty(tokens, hq, DIM, dtype=torch.bfloat16, device=DEV))
    return s


def _prepare_pages(case, rng, randn):
    """Prompts in the first rows, their samples (forked once already) in the rows after them."""
    g, n = case["groups"], case["samples"]
    prompt = rng.permutation(_spread(case["ctx_lo"], case["ctx_hi"], g))
    rows = g + g * n
    have = (prompt + PAGE - 1) // PAGE
    pages = int(have.sum()) + 2 * g * n + 5
    ids = rng.permutation(pages).astype(np.int32)
    table = np.full((rows, int(have.max()) + 2), -1, np.int32)
    table[:g][np.arange(table.shape[1])[None, :] < have[:, None]] = ids[: int(have.sum())]
    refs = np.zeros(pages, np.int32)
    src = np.repeat(np.arange(g), n)
    dst = g + np.arange(g * n)
    used = int(have.sum())
    # the samples of the round before: the prompt's full pages, a tail page and one page more
    full = prompt[src] // PAGE
    keep = np.arange(table.shape[1])[None, :] < full[:, None]
    table[dst] = np.where(keep, table[src], -1)
    np.add.at(refs, table[dst][keep], 1)
    table[dst, full] = ids[used:used + g * n]
    longer = rng.random(g * n) < 0.5
    more = int(longer.sum())
    table[dst[longer], full[longer] + 1] = ids[used + g * n: used + g * n + more]
    free = np.zeros(pages, np.int32)
    left = ids[used + g * n + more:]
    free[: len(left)] = left
    lens = np.concatenate([prompt, prompt[src]])
    s = dict(case=case, kind="pages", bt=_put(table), sl=_put(lens), refs=_put(refs), free=_put(free),
             count=_put([len(left)]), keep=_put(np.where(np.arange(rows) < g, lens, 0)), src=_put(src), dst=_put(dst),
             copy_src=_put(np.full(g * n, -1)), copy_dst=_put(np.full(g * n, -1)),
             scratch=torch.zeros(64, dtype=torch.int32, device=DEV),
             status=torch.zeros(1, dtype=torch.int32, device=DEV),
             pools=randn(2 * case["layers"], pages, case["hkv"], PAGE, DIM))
    if own:
        from paper_2608_22167_gb300 import mcpu
        s["list"] = mcpu.PoolList([s["pools"][i] for i in range(s["pools"].shape[0])])
    return s


# -------------------------------------------------------------------- a pass
def run(s):
    return (_own if own else _plain)[s["kind"]](s)


def _own_norm(s):
    from paper_2608_22167_gb300 import mcpu
    mcpu.mcpu_norm_rope_kv_append(s["q"], s["k"], s["v"], s["wq"], s["wk"], s["eps"], s["positions"], s["rope"],
                                  s["q_out"], s["kc"], s["vc"], s["bt"], s["sl"], s["qsl"], s["status"])
    return dict(q=s["q_out"], k=s["kc"], v=s["vc"])


def _own_tree(s):
    from paper_2608_22167_gb300 import mcpu
    mcpu.mcpu_tree_attention_forward(s["q"], s["kc"], s["vc"], s["bt"], s["sl"], s["qsl"], s["mask"], s["positions"],
                                     s["window"], s["scale"], s["out"], s["lse"], s["ws"], sinks=s["sinks"])
    return dict(out=s["out"], lse=s["lse"])


def _own_compact(s):
    from paper_2608_22167_gb300 import mcpu
    mcpu.mcpu_compact_kv(s["list"], s["bt"], s["sl"], s["qsl"], s["path"], s["taken"], s["new_sl"], s["status"])
    return dict(pools=s["pools"], seq_lens=s["new_sl"])


def _own_pages(s):
    from paper_2608_22167_gb300 import mcpu
    mcpu.mcpu_shrink_block_tables(s["bt"], s["keep"], 0, s["refs"], s["free"], s["count"], s["scratch"], s["status"])
    mcpu.mcpu_fork_block_tables(s["bt"], s["sl"], s["src"], s["dst"], s["refs"], s["free"], s["count"], s["copy_src"],
                                s["copy_dst"], s["scratch"], s["status"])
    mcpu.mcpu_copy_pages(s["list"], s["copy_src"], s["copy_dst"], s["status"])
    return _pages_out(s)


def _pages_out(s):
    return dict(table=s["bt"], seq_lens=s["sl"], refs=s["refs"], free=s["free"], count=s["count"], pools=s["pools"])


def _row_of_token(s):
    t = torch.arange(s["q"].shape[0], device=DEV)
    r = torch.searchsorted(s["qsl"], t.int(), right=True) - 1
    return r, t - s["qsl"][r]


def _plain_norm(s):
    r, i = _row_of_token(s)
    slot = s["sl"][r] - (s["qsl"][r + 1] - s["qsl"][r]) + i
    angle = s["rope"][slot if s["positions"] is None else s["positions"].long()][:, None, :]
    cos, sin = angle[..., :DIM // 2], angle[..., DIM // 2:]

    def turn(x, w):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * w
        a, b = x[..., :DIM // 2], x[..., DIM // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(torch.bfloat16)

    s["q_out"].copy_(turn(s["q"], s["wq"]))
    page = s["bt"][r, slot // PAGE].long()
    s["kc"][page, :, slot % PAGE] = turn(s["k"], s["wk"])
    s["vc"][page, :, slot % PAGE] = s["v"]
    return dict(q=s["q_out"], k=s["kc"], v=s["vc"])


def _plain_tree(s):
    # every row padded to the most nodes and to the widest span of keys from its first visible page
    case, most, rows = s["case"], s["most"], s["rows"]
    hq, hkv = case["hq"], case["hkv"]
    g = hq // hkv
    r, i = _row_of_token(s)
    lens = s["qsl"][1:] - s["qsl"][:-1]
    ctx = s["sl"] - lens
    first = (ctx - s["window"] + 1).clamp(min=0) // PAGE if s["window"] > 0 else torch.zeros_like(ctx)
    span = (s["span"] + PAGE - 1) // PAGE
    at = first[:, None] + torch.arange(span, device=DEV)[None, :]
    page = torch.gather(s["bt"], 1, at.clamp(max=s["bt"].shape[1] - 1).long()).clamp(min=0).long()
    k, v = (x[page].transpose(2, 3).reshape(rows, span * PAGE, hkv, DIM).transpose(1, 2).float()
            for x in (s["kc"], s["vc"]))
    q = torch.zeros(rows, most, hq, DIM, device=DEV)
    q[r, i] = s["q"].float()
    q = q.view(rows, most, hkv, g, DIM).permute(0, 2, 1, 3, 4).reshape(rows, hkv, most * g, DIM)
    key = (first * PAGE)[:, None] + torch.arange(span * PAGE, device=DEV)[None, :]  # position of each gathered key
    node = (key - ctx[:, None])[r]  # its number among the row's nodes, below 0 in the context
    word = torch.gather(s["mask"], 1, (node // 32).clamp(0, s["mask"].shape[1] - 1).long())
    sees = torch.where(node < 0, torch.ones_like(word), (word >> (node % 32)) & 1) != 0
    sees &= node < lens[r][:, None]
    if s["window"] > 0:
        sees &= (node >= 0) | (s["positions"][:, None] - key[r] < s["window"])
    full = torch.zeros(rows, most, span * PAGE, dtype=torch.bool, device=DEV)
    full[r, i] = sees
    full = full[:, None, :, None, :].expand(rows, 1, most, g, span * PAGE).reshape(rows, 1, most * g, span * PAGE)
    x = torch.matmul(q, k.transpose(2, 3)) * s["scale"]
    x = x.masked_fill_(~full, -math.inf)
    top = x.amax(-1, keepdim=True)
    if s["sinks"] is not None:
        sink = s["sinks"].view(1, hkv, 1, g, 1).expand(rows, hkv, most, g, 1).reshape(rows, hkv, most * g, 1)
        top = torch.maximum(top, sink)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    x = x.sub_(top).exp_()
    z = x.sum(-1, keepdim=True)
    if s["sinks"] is not None:
        z = z + torch.exp(sink - top)
    o = torch.matmul(x, v) / torch.where(z == 0, torch.ones_like(z), z)
    lse = top + torch.log(z)

    def back(y):
        return y.reshape(rows, hkv, most, g, -1).permute(0, 2, 1, 3, 4).reshape(rows, most, hq, -1)[r, i]

    s["out"].copy_(back(o))
    s["lse"].copy_(back(lse)[..., 0])
    return dict(out=s["out"], lse=s["lse"])


def _plain_compact(s):
    lens = s["qsl"][1:] - s["qsl"][:-1]
    ctx = s["sl"] - lens
    r, i = (torch.arange(s["path"].shape[1], device=DEV)[None, :] < s["taken"][:, None]).nonzero(as_tuple=True)
    old, new = (ctx[r] + s["path"][r, i]).long(), ctx[r] + i
    rows = s["pools"][:, s["bt"][r, old // PAGE].long(), :, old % PAGE]
    s["pools"][:, s["bt"][r, new // PAGE].long(), :, new % PAGE] = rows
    s["new_sl"].copy_(ctx + s["taken"])
    return dict(pools=s["pools"], seq_lens=s["new_sl"])


def _plain_pages(s):
    bt, refs, free, count = s["bt"], s["refs"], s["free"], s["count"]
    j = torch.arange(bt.shape[1], device=DEV)[None, :]
    # release what lies past the kept lengths; pages without another holder return to the stack, by number
    drop = (j >= ((s["keep"] + PAGE - 1) // PAGE)[:, None]) & (bt >= 0)
    refs -= torch.bincount(bt[drop].long(), minlength=refs.shape[0])
    gone = (refs < 0).nonzero()[:, 0]
    free[count.long() + torch.arange(gone.shape[0], device=DEV)] = gone.int()
    count += gone.shape[0]
    refs[gone] = 0
    bt[drop] = -1
    # fork: full pages shared, a fresh page for a partial tail
    src, dst = s["src"].long(), s["dst"].long()
    lens = s["sl"][src]
    full = (lens // PAGE)[:, None]
    bt[dst] = torch.where(j < full, bt[src], torch.full_like(bt[src], -1))
    shared = bt[dst]
    refs += torch.bincount(shared[shared >= 0].long(), minlength=refs.shape[0])
    part = (lens % PAGE != 0).nonzero()[:, 0]
    page = free[count.long() - 1 - torch.arange(part.shape[0], device=DEV)]
    count -= part.shape[0]
    tail = (lens[part] // PAGE).long()
    s["copy_src"].fill_(-1)
    s["copy_dst"].fill_(-1)
    s["copy_src"][part] = bt[src[part], tail]
    s["copy_dst"][part] = page
    bt[dst[part], tail] = page
    s["sl"][dst] = lens
    # the tail pages' contents, in every layer
    s["pools"][:, page.long()] = s["pools"][:, bt[src[part], tail].long()]
    return _pages_out(s)


_own = dict(norm=_own_norm, tree=_own_tree, compact=_own_compact, pages=_own_pages)
_plain = dict(norm=_plain_norm, tree=_plain_tree, compact=_plain_compact, pages=_plain_pages)


# ---------------------------------------------------------------------- work
def work(case):
    hkv = case["hkv"]
    row = 2 * DIM  # bytes of one head's key or value
    if case["kind"] == "pages":
        g, n = case["groups"], case["samples"]
        prompt = _spread(case["ctx_lo"], case["ctx_hi"], g)
        partial = n * int((prompt % PAGE != 0).sum())
        entries = n * int(((prompt + PAGE - 1) // PAGE).sum())
        # tail pages read and written in every pool; each sample's entries released (table and count) and set again
        return dict(bytes=partial * 2 * case["layers"] * hkv * PAGE * row * 2 + entries * 4 * 6, flops=0)
    rng = np.random.default_rng(5)
    ctx, lens = _lengths(case, rng)
    tokens = int(lens.sum())
    if case["kind"] == "norm":
        heads = case["hq"] + 2 * hkv
        return dict(bytes=tokens * heads * row * 2 + tokens * DIM * 4, flops=tokens * (case["hq"] + hkv) * DIM * 8)
    if case["kind"] == "compact":
        # on average half of the longest path is accepted, and most of it lies elsewhere
        most = min(6, int(lens.max()))
        moved = float(np.minimum(np.arange(most + 1)[:, None], lens[None, :]).mean(0).sum())
        return dict(bytes=moved * 2 * case["layers"] * hkv * row * 2, flops=0)
    keys = np.minimum(ctx, case["window"] - 1) if case["window"] > 0 else ctx
    pairs = float((keys * lens).sum()) + float((lens * np.minimum(lens, 8)).sum() / 2)
    hq = case["hq"]
    return dict(bytes=float((keys + lens).sum()) * 2 * hkv * row + tokens * hq * (2 * row + 4), flops=pairs * hq * 4 * DIM)


# --------------------------------------------------------------------- exact
def exact(case, seed):
    s = prepare(case, seed)
    return dict(norm=_exact_norm, tree=_exact_tree, compact=_exact_compact, pages=_exact_pages)[s["kind"]](s)


def _slots(s, r):
    """Page and slot of every token of row r that the table holds, by position."""
    n = int(s["sl"][r])
    pos = torch.arange(n, device=DEV)
    return s["bt"][r].long()[pos // PAGE], pos % PAGE


def _exact_norm(s):
    kc, vc = s["kc"].double(), s["vc"].double()
    qsl, sl = s["qsl"].tolist(), s["sl"].tolist()
    parts = []
    for r in range(s["rows"]):
        a, b = qsl[r], qsl[r + 1]
        page, slot = (x[sl[r] - (b - a):] for x in _slots(s, r))
        pos = s["positions"][a:b].long() if s["positions"] is not None else torch.arange(sl[r] - (b - a), sl[r], device=DEV)
        half = s["rope"][pos].double()
        unit = torch.complex(half[:, :DIM // 2], half[:, DIM // 2:])[:, None]

        def turned(x, w):
            x = x.double()
            x = x / x.square().mean(2, keepdim=True).add(s["eps"]).sqrt() * w.double()
            z = torch.complex(x[..., :DIM // 2].contiguous(), x[..., DIM // 2:].contiguous()) * unit
            return torch.cat([z.real, z.imag], 2)

        parts.append(turned(s["q"][a:b], s["wq"]))
        kc[page, :, slot] = turned(s["k"][a:b], s["wk"])
        vc[page, :, slot] = s["v"][a:b].double()
    return dict(q=torch.cat(parts), k=kc, v=vc)


def _exact_tree(s):
    hq, hkv = s["case"]["hq"], s["case"]["hkv"]
    qsl, sl = s["qsl"].tolist(), s["sl"].tolist()
    outs, lses = [], []
    for r in range(s["rows"]):
        a, b = qsl[r], qsl[r + 1]
        n = b - a
        ctx = sl[r] - n
        low = max(0, ctx - s["window"] + 1) if s["window"] > 0 else 0
        page, slot = (x[low:] for x in _slots(s, r))
        k, v = s["kc"][page, :, slot].double(), s["vc"][page, :, slot].double()  # [keys, hkv, dim]
        words = s["mask"][a:b].long() & 0xFFFFFFFF
        anc = torch.stack([(words[:, j // 32] >> (j % 32)) & 1 for j in range(n)], 1).bool()  # [node, node]
        pos = torch.arange(low, ctx, device=DEV)
        near = torch.ones(n, ctx - low, dtype=torch.bool, device=DEV)
        if s["window"] > 0:
            near = s["positions"][a:b, None] - pos[None] < s["window"]
        sees = torch.cat([near, anc], 1)
        o = torch.empty(n, hq, DIM, dtype=torch.float64, device=DEV)
        e = torch.empty(n, hq, dtype=torch.float64, device=DEV)
        for h in range(hkv):
            heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            x = torch.einsum("nhd,kd->nhk", s["q"][a:b, heads].double(), k[:, h]) * s["scale"]
            x = torch.where(sees[:, None], x, -math.inf)
            if s["sinks"] is not None:
                x = torch.cat([x, s["sinks"][heads].double()[None, :, None].expand(n, -1, 1)], 2)
            e[:, heads] = torch.logsumexp(x, 2)
            w = torch.softmax(x, 2).nan_to_num(0.0)[:, :, : k.shape[0]]
            o[:, heads] = torch.einsum("nhk,kd->nhd", w, v[:, h])
        outs.append(o)
        lses.append(e)
    return dict(out=torch.cat(outs), lse=torch.cat(lses))


def _exact_compact(s):
    pools = s["pools"].double()
    path, taken, qsl, sl = (s[k].tolist() for k in ("path", "taken", "qsl", "sl"))
    bt = s["bt"].tolist()
    old, new = [], []
    for r in range(s["rows"]):
        base = sl[r] - (qsl[r + 1] - qsl[r])
        for i in range(taken[r]):
            p = base + path[r][i]
            old.append((bt[r][p // PAGE], p % PAGE))
            new.append((bt[r][(base + i) // PAGE], (base + i) % PAGE))
    if old:
        (op, os_), (np_, ns) = (torch.tensor(x, device=DEV).T for x in (old, new))
        pools[:, np_, :, ns] = pools[:, op, :, os_].clone()
    return dict(pools=pools, seq_lens=None)


def _exact_pages(s):
    # the page numbers are whole and compared as such; what the forks' tail pages hold is the prompts' tails
    table, refs, free = s["bt"].tolist(), s["refs"].tolist(), s["free"].tolist()[: int(s["count"])]
    keep, lens = s["keep"].tolist(), s["sl"].tolist()
    gone = []
    for r, row in enumerate(table):
        for j in range(-(-keep[r] // PAGE), len(row)):
            if row[j] >= 0:
                refs[row[j]] -= 1
                gone += [row[j]] if refs[row[j]] < 0 else []
    free += sorted(gone)
    old, new = [], []
    for src in s["src"].tolist():
        if lens[src] % PAGE:
            old.append(table[src][lens[src] // PAGE])
            new.append(free.pop())
    pools = s["pools"].double()
    if old:
        pools[:, torch.tensor(new, device=DEV)] = pools[:, torch.tensor(old, device=DEV)].clone()
    return dict(table=None, seq_lens=None, refs=None, free=None, count=None, pools=pools)
