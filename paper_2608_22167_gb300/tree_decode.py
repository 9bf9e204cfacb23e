"""Tree-drafted decoding over a paged cache, with every step on the device.

``PagedCache`` owns the KV pools of the layers that share one block table,
the table, the pages' holder counts and the stack of free pages; its methods
are the calls of one round (no host round trip, capturable in a CUDA graph as
long as the tensors stay the same):

    cache.extend(new_lens)              pages for the drafted tokens
    q = cache.append(layer, ...)        norm, rotation, K/V to the pages
    cache.attend(layer, q, ...)         every node over the context and its ancestors
    path, path_len, ... = cache.verify(logits, ...)   which drafted tokens are accepted
    cache.keep(qsl, path, path_len)     the accepted path stays, spare pages return
    cache.evict(budget, ...)            rows past a limit cut to the keys that got most attention
    cache.fork(src, dst)                new samples from running rows
    cache.drop(rows)                    rows leave

``python -m paper_2608_22167_gb300.tree_decode`` runs a toy model (random
weights, two layers) with forked samples: it decodes greedily with drafted
trees and reports the tokens accepted a round, then samples on in a cache that
is held to a budget of keys. No model of any framework is loaded; PyTorch does
the toy model's projections.
"""
from __future__ import annotations

from bisect import bisect_left, insort

import torch

from . import mcpu

PAGE, HEAD_DIM = 16, 64


def _span(x):
    """Where a dense tensor lies."""
    return x.data_ptr(), x.data_ptr() + x.numel() * x.element_size()


class PagedCache:
    """The pools, table, page counts and stack of layers that share a block table. sliding_window > 0: all of them
    attend within that window, and `keep` returns the pages before it. count_weights: `keep` (or `observe`) counts the
    attention that every key got, for `evict`; `attend` keeps hold of each layer's q and log-sum-exps until then, so
    they are not to be written before, and layers do not share them."""

    def __init__(self, layers, rows, max_pages, num_pages, num_q_heads, num_kv_heads, device="cuda", sliding_window=0,
                 count_weights=False):
        shape = (num_pages, num_kv_heads, PAGE, HEAD_DIM)
        i32 = dict(dtype=torch.int32, device=device)
        self.k = [torch.empty(shape, dtype=torch.bfloat16, device=device) for _ in range(layers)]
        self.v = [torch.empty(shape, dtype=torch.bfloat16, device=device) for _ in range(layers)]
        self.pools = mcpu.PoolList(self.k + self.v)
        self.num_q_heads, self.rows, self.sliding_window = num_q_heads, rows, sliding_window
        self.block_table = torch.full((rows, max_pages), -1, **i32)
        self.seq_lens = torch.zeros(rows, **i32)
        self.new_lens = torch.zeros(rows, **i32)
        self.held_lens = torch.zeros(rows, **i32)  # lengths whose pages the rows were left with: not grown again
        self.page_refs = torch.zeros(num_pages, **i32)
        self.free_pages = torch.arange(num_pages, **i32)
        self.free_count = torch.tensor([num_pages], **i32)
        self.page_scratch = torch.zeros(mcpu.PAGE_SCRATCH, **i32)
        d = mcpu.Dims(rows, 0, max_pages, num_pages, num_q_heads, num_kv_heads, HEAD_DIM, PAGE)
        self.workspace = mcpu.new_tree_workspace(d, device)
        self.status = mcpu.status_word(self.workspace)
        self.evicted = torch.zeros(rows, **i32)  # keys that a row has lost: its slot s holds no earlier position than s + evicted
        self.key_weights = self.weights_workspace = None
        self.asked = [None] * layers  # (q, lse, scale, window) of each layer's last attention, if weights are counted,
        self.spans = []               # and where its tensors lie: (begin, end, layer), ascending
        if count_weights:
            if sliding_window > 0:
                raise ValueError("the keys of a sliding window are let go by their age")
            self.key_weights = torch.zeros(layers, rows, num_kv_heads, max_pages * PAGE, device=device)
            self.weights_workspace = mcpu.new_weights_workspace(d, device)

    def check(self):
        """Raises if a call so far has reported a device-side error (synchronises)."""
        for ws in (self.workspace, self.weights_workspace):
            code, bits = mcpu.mcpu_read_device_status(ws) if ws is not None else (0, 0)
            if code:
                raise mcpu.McpuError(code, f"device status bits {bits}")

    def extend(self, new_lens):
        """Row lengths after the next append (int32 [rows]) and the pages for them. What is appended follows the tokens
        that a row holds: pages before that may be shared with other rows."""
        self._let_go()
        self.seq_lens.copy_(new_lens)
        mcpu.mcpu_grow_block_tables_from(self.block_table, self.seq_lens, self.held_lens, self.free_pages,
                                         self.free_count, self.status)

    def append(self, layer, q, k, v, q_weight, k_weight, eps, cos_sin, query_start_loc, positions=None, q_out=None):
        """Norm, rotation and KV append of a layer's projected q, k and v; returns the rotated q."""
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        else:
            self._not_held(layer, q_out)
        mcpu.mcpu_norm_rope_kv_append(q, k, v, q_weight, k_weight, eps, positions, cos_sin, q_out, self.k[layer],
                                      self.v[layer], self.block_table, self.seq_lens, query_start_loc, self.status)
        return q_out

    def attend(self, layer, q, query_start_loc, tree_mask, positions=None, sliding_window=None,
               scale=HEAD_DIM ** -0.5, sinks=None, out=None, lse=None):
        """Attention of every node over its row's context (in the cache's window, if none is given) and the nodes
        its mask names: in a window the mask has to keep to it too (tree_masks)."""
        sliding_window = self.sliding_window if sliding_window is None else sliding_window
        self._not_held(layer, q, lse, out)
        if out is not None and self.key_weights is not None and _span(out)[0] < _span(q)[1] and _span(q)[0] < _span(out)[1]:
            raise ValueError("the output may not take the place of q, whose attention is yet to be counted")
        out = torch.empty_like(q) if out is None else out
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device) if lse is None else lse
        mcpu.mcpu_tree_attention_forward(q, self.k[layer], self.v[layer], self.block_table, self.seq_lens,
                                         query_start_loc, tree_mask, positions, sliding_window, scale, out, lse,
                                         self.workspace, sinks=sinks)
        if self.key_weights is not None:
            self._hold(layer, q, lse, scale, sliding_window)
        return out, lse

    def verify(self, logits, tokens, parents, query_start_loc, max_accept, temperature=None, draft_logits=None,
               uniforms=None, exponentials=None):
        """Which nodes of each row's tree are accepted, from the target's logits at every node: path [rows,
        max_accept], path_len, the token after it, and the log-probabilities of what is emitted. temperature (float32
        [rows], 0: greedy) None: all greedy. Random numbers that are not given are drawn."""
        dev, rows = logits.device, self.rows
        i32 = dict(dtype=torch.int32, device=dev)
        path, path_len, token = torch.empty(rows, max_accept, **i32), torch.empty(rows, **i32), torch.empty(rows, **i32)
        logprobs = torch.empty(rows, max_accept, device=dev)
        if temperature is not None:
            if uniforms is None:
                uniforms = torch.rand(logits.shape[0], device=dev)
            if exponentials is None:  # (never 0, of which only rounding could make one)
                exponentials = torch.empty(rows, logits.shape[1], device=dev).exponential_().clamp_(min=1e-30)
        mcpu.mcpu_verify_tree(logits, tokens, parents, query_start_loc, temperature, uniforms, exponentials, path, path_len,
                              token, logprobs, self.status, draft_logits=draft_logits)
        return path, path_len, token, logprobs

    def observe(self, query_start_loc, path=None, path_len=None, decay=1.0):
        """Counts the attention of the last step's queries (those of the accepted nodes, once `keep` has moved their
        keys; None: all) for every layer; earlier weights are multiplied by decay. Before `extend` or `evict`, which
        change what the queries saw."""
        self._check_counted()
        for layer, (q, lse, scale, window) in enumerate(self.asked):
            mcpu.mcpu_accumulate_weights(q, lse, self.k[layer], self.block_table, self.seq_lens, query_start_loc, window,
                                         scale, decay, self.key_weights[layer], self.weights_workspace, query_path=path,
                                         path_len=path_len)
        self._let_go()

    def evict(self, budget, keep_first=4, keep_last=32, limit=None):
        """Rows of more than `limit` keys (None: budget) are cut to budget: the first, the last, and those that got
        most attention, for every kv head of every layer by itself. Rows that share pages from keep_first on are left
        alone and reported, which `check` tells from then on (their forks would lose the keys too): with a common
        prompt keep_first reaches to the end of its full pages. Positions go on from `seq_lens + evicted`. Layers with a window of at
        most keep_last stay right, since the last keys stay next to each other: `attend` is given positions less
        `evicted` there, which are the slots that the window counts."""
        if self.key_weights is None:
            raise ValueError("keys are evicted by the weights of a cache made with count_weights")
        mcpu.mcpu_evict_kv(self.pools, self.key_weights, self.block_table, self.seq_lens, budget if limit is None else limit,
                           budget, keep_first, keep_last, self.key_weights, self.new_lens, self.status,
                           page_refs=self.page_refs)
        self._let_go()
        self.evicted += self.seq_lens - self.new_lens
        self.seq_lens.copy_(self.new_lens)
        self._release(self.seq_lens)

    def keep(self, query_start_loc, path, path_len, decay=1.0):
        """Keeps the accepted nodes path[r, :path_len[r]] of each row's tree, in every layer, counts their attention
        if weights are counted, and returns the pages behind them."""
        if self.key_weights is not None:
            self._check_counted()
        mcpu.mcpu_compact_kv(self.pools, self.block_table, self.seq_lens, query_start_loc, path, path_len,
                             self.new_lens, self.status)
        self.seq_lens.copy_(self.new_lens)
        if self.key_weights is not None:
            self.observe(query_start_loc, path, path_len, decay)
        self.held_lens.copy_(self.seq_lens)
        self._release(self.seq_lens, self.sliding_window)

    def fork(self, src_rows, dst_rows):
        """Rows dst_rows (empty) become copies of src_rows: full pages shared, partial last pages copied. Not between
        a row's `append` and its `keep`, which moves rows inside pages that would be shared by then. Pairs that do not
        name two rows are skipped and reported."""
        n = src_rows.shape[0]
        if self.key_weights is not None and n > 0:
            # what the kernel skips does as the first pair that it does not, or (none) copies row 0 to itself
            src, dst = src_rows.long(), dst_rows.long()
            lens = self.seq_lens[src.clamp(0, self.rows - 1)]
            pair = (src >= 0) & (src < self.rows) & (dst >= 0) & (dst < self.rows) & (src != dst) & (lens >= 0) & \
                (lens <= self.block_table.shape[1] * PAGE)
            first = pair.int().argmax().expand(1)
            some = pair.any()
            src = torch.where(pair, src, torch.where(some, src[first], 0))
            dst = torch.where(pair, dst, torch.where(some, dst[first], 0))
        copy = torch.empty(2, n, dtype=torch.int32, device=src_rows.device)
        mcpu.mcpu_fork_block_tables(self.block_table, self.seq_lens, src_rows, dst_rows, self.page_refs,
                                    self.free_pages, self.free_count, copy[0], copy[1], self.page_scratch, self.status)
        mcpu.mcpu_copy_pages(self.pools, copy[0], copy[1], self.status)
        if self.key_weights is not None and n > 0:
            self.evicted[dst] = self.evicted[src]
            self.key_weights[:, dst] = self.key_weights[:, src]
        self.held_lens.copy_(self.seq_lens)

    def drop(self, rows):
        """Frees the rows (int64 indices)."""
        self.seq_lens[rows] = 0
        if self.key_weights is not None:
            self.evicted[rows] = 0
            self.key_weights[:, rows] = 0  # the slots of rows to come start without weights
        self._release(self.seq_lens)

    def _hold(self, layer, q, lse, scale, sliding_window):
        self.asked[layer] = (q, lse, scale, sliding_window)
        self.spans = [s for s in self.spans if s[2] != layer]
        for x in (q, lse):
            insort(self.spans, (*_span(x), layer))

    def _not_held(self, layer, *tensors):
        """Refuses buffers that hold what another layer's attention is yet to be counted from."""
        for x in tensors if self.spans else ():
            if x is None or x.numel() == 0:
                continue
            begin, end = _span(x)
            for s in self.spans[max(bisect_left(self.spans, (begin,)) - 1, 0):]:
                if s[0] >= end:
                    break
                if s[1] > begin and s[2] != layer:
                    raise ValueError("each layer needs q and log-sum-exps of its own until their attention is counted")

    def _check_counted(self):
        if self.key_weights is None:
            raise ValueError("attention is counted by a cache made with count_weights")
        if None in self.asked:
            raise ValueError(f"layer {self.asked.index(None)} has not attended since the last step was counted")

    def _let_go(self):
        """What was held is counted, or can be no more."""
        self.asked = [None] * len(self.k)
        self.spans = []

    def _release(self, lens, sliding_window=0):
        torch.minimum(self.held_lens, lens, out=self.held_lens)
        mcpu.mcpu_shrink_block_tables(self.block_table, lens, sliding_window, self.page_refs, self.free_pages,
                                      self.free_count, self.page_scratch, self.status)


def tree_masks(parents, sliding_window=0):
    """Ancestor masks (int32 [nodes, words]) and depths of trees given as lists of parents (-1: the context),
    nodes in topological order: host tensors to copy to the device. The masks are all that tree attention knows of
    the nodes: for a layer with a sliding window, give the window here too, and a node's mask holds itself and the
    ancestors less than the window above it only."""
    words = max(1, (max((len(p) for p in parents), default=1) + 31) // 32)
    masks, depths = [], []
    for parent in parents:
        rows, depth = [], []
        near = []  # each node's ancestors inside the window, then itself
        for i, up in enumerate(parent):
            if not -1 <= up < i:
                raise ValueError("a node comes after its parent")
            bits = (rows[up] if up >= 0 else 0) | 1 << i
            if sliding_window > 0:
                near.append((near[up] if up >= 0 else []) + [i])
                if len(near[i]) > sliding_window:
                    bits &= ~(1 << near[i].pop(0))
            rows.append(bits)
            depth.append(depth[up] + 1 if up >= 0 else 0)
        masks += [[(b >> 32 * w & 0xFFFFFFFF) - (1 << 32 if b >> 32 * w & 1 << 31 else 0) for w in range(words)]
                  for b in rows]
        depths += depth
    return torch.tensor(masks, dtype=torch.int32).view(-1, words), torch.tensor(depths, dtype=torch.int32)


def rope_table(max_position, base=150000.0, device="cuda"):
    """cos then sin of position * base^(-2i / 64): float32 [max_position, 64]."""
    i = torch.arange(HEAD_DIM // 2, device=device, dtype=torch.float64)
    angle = torch.arange(max_position, device=device, dtype=torch.float64)[:, None] * base ** (-2 * i / HEAD_DIM)
    return torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()


class ToyModel:
    """A small decoder with random weights: what the example and its test put around the cache."""

    def __init__(self, layers=2, num_q_heads=8, num_kv_heads=2, vocab=12, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        width = num_q_heads * HEAD_DIM

        def w(*shape):
            return torch.randn(shape, generator=g, device=device, dtype=torch.bfloat16)

        self.hq, self.hkv, self.vocab = num_q_heads, num_kv_heads, vocab
        self.embed, self.head = w(vocab, width), w(width, vocab)
        self.qkv = [w(width, (num_q_heads + 2 * num_kv_heads) * HEAD_DIM) / width ** 0.5 for _ in range(layers)]
        self.o = [w(width, width) / width ** 0.5 for _ in range(layers)]
        self.norm = [(1 + 0.2 * torch.randn(2, HEAD_DIM, generator=g, device=device)).contiguous() for _ in range(layers)]
        self.cos_sin = rope_table(4096, device=device)

    def run(self, cache, tokens, query_start_loc, mask, positions):
        """Logits of every query token (its nodes appended to the cache)."""
        x = self.embed[tokens]
        for i, (qkv, o, norm) in enumerate(zip(self.qkv, self.o, self.norm)):
            h = torch.nn.functional.layer_norm(x.float(), x.shape[-1:]).to(x.dtype) @ qkv
            q, k, v = (t.unflatten(1, (-1, HEAD_DIM)) for t in h.split(
                [self.hq * HEAD_DIM, self.hkv * HEAD_DIM, self.hkv * HEAD_DIM], dim=1))
            q = cache.append(i, q, k, v, norm[0], norm[1], 1e-6, self.cos_sin, query_start_loc, positions)
            a, _ = cache.attend(i, q, query_start_loc, mask, positions)
            x = x + a.flatten(1) @ o
        return torch.nn.functional.layer_norm(x.float(), x.shape[-1:]) @ self.head.float()


def accept_greedy(parents, tokens, choice):
    """The accepted path of one tree: from the root (node 0, the last token of the row) down to the children
    whose token is the model's choice at their parent; and the model's next token."""
    path, at = [0], 0
    while True:
        nxt = next((i for i in range(at + 1, len(parents)) if parents[i] == at and tokens[i] == choice[at]), None)
        if nxt is None:
            return path, int(choice[at])
        path.append(nxt)
        at = nxt


def generate(model, cache, last, rounds, seed=0, nodes=24, temperature=0.0, budget=0, keep_first=4, keep_last=32):
    """Decoding of the rows whose last tokens (not yet in the cache) are `last`, `rounds` rounds with a drafted tree
    each: node 0 is the last token, the others random drafts. Greedy at temperature 0, else sampled. budget > 0: rows
    are cut to so many keys once a round (the cache counts weights). Returns each row's new tokens."""
    g = torch.Generator()
    g.manual_seed(seed)
    rows = len(last)
    dev = cache.block_table.device
    draws = torch.Generator(device=dev)
    draws.manual_seed(seed)
    made = [[] for _ in range(rows)]
    heat = torch.full((rows,), float(temperature), device=dev) if temperature > 0 else None
    qsl = torch.arange(0, rows * nodes + 1, nodes, dtype=torch.int32, device=dev)
    for _ in range(rounds):
        parents = [[-1] + [int(torch.randint(max(0, i - 6), i, (1,), generator=g)) for i in range(1, nodes)]
                   for _ in range(rows)]
        tokens = [[last[r]] + torch.randint(0, model.vocab, (nodes - 1,), generator=g).tolist() for r in range(rows)]
        mask, depth = tree_masks(parents)
        tree = torch.tensor(parents, dtype=torch.int32, device=dev).flatten()
        nodes_tokens = torch.tensor(tokens, device=dev).flatten()
        ctx = cache.seq_lens.clone()
        positions = ((ctx + cache.evicted).repeat_interleave(nodes) + depth.to(dev)).int()
        cache.extend(ctx + nodes)
        logits = model.run(cache, nodes_tokens, qsl, mask.to(dev), positions)
        uniforms = exponentials = None
        if heat is not None:
            uniforms = torch.rand(rows * nodes, generator=draws, device=dev)
            exponentials = torch.empty(rows, model.vocab, device=dev).exponential_(generator=draws).clamp_(min=1e-30)
        path, path_len, token, _ = cache.verify(logits, nodes_tokens.int(), tree, qsl, nodes, heat, uniforms=uniforms,
                                                exponentials=exponentials)
        cache.keep(qsl, path, path_len)
        if budget > 0:
            cache.evict(budget, keep_first, keep_last)
        last[:] = token.tolist()
        for r, (way, n) in enumerate(zip(path.tolist(), path_len.tolist())):
            made[r] += [tokens[r][i] for i in way[1:n]] + [last[r]]
    cache.check()
    return made


def main():
    model = ToyModel()
    prompts, samples = 4, 4
    rows = prompts * (1 + samples)
    # the prompts: chains of 37 to 100 tokens in the first rows, then four samples of each
    lens = [37, 64, 81, 100]
    mask, depth = tree_masks([list(range(-1, n - 1)) for n in lens])
    qsl = torch.tensor([0] + [sum(lens[:i + 1]) for i in range(prompts)] + [sum(lens)] * (rows - prompts),
                       dtype=torch.int32, device="cuda")
    tokens = torch.randint(0, model.vocab, (sum(lens),), device="cuda")

    def fill(cache):
        cache.extend(torch.tensor(lens + [0] * (rows - prompts), device="cuda"))
        model.run(cache, tokens, qsl, mask.cuda(), depth.cuda())

    cache = PagedCache(2, rows, 64, 1200, model.hq, model.hkv)
    fill(cache)
    src = torch.arange(prompts, dtype=torch.int32, device="cuda").repeat_interleave(samples)
    dst = torch.arange(prompts, rows, dtype=torch.int32, device="cuda")
    cache.fork(src, dst)
    cache.check()
    free = int(cache.free_count)
    rounds = 20
    made = generate(model, cache, [r % model.vocab for r in range(rows)], rounds)
    n = sum(map(len, made))
    print(f"{rows} rows, {rounds} rounds: {n} tokens, {n / rows / rounds:.2f} a row and round; "
          f"{free - int(cache.free_count)} pages taken since the fork")
    cache.drop(torch.arange(rows, device="cuda"))
    cache.check()
    assert int(cache.free_count) == cache.page_refs.shape[0] and not cache.page_refs.any()

    # the prompts alone, sampled on with at most 96 keys a head
    cache = PagedCache(2, rows, 64, 1200, model.hq, model.hkv, count_weights=True)
    fill(cache)
    cache.observe(qsl)
    cache.held_lens.copy_(cache.seq_lens)
    made = generate(model, cache, [r % model.vocab for r in range(rows)], 2 * rounds, temperature=0.8, budget=96)
    n = sum(map(len, made))
    print(f"sampled with 96 keys a head: {n} tokens, {n / rows / (2 * rounds):.2f} a row and round; "
          f"{int(cache.evicted.sum())} keys let go, rows of {int(cache.seq_lens.max())} keys at most")
    cache.drop(torch.arange(rows, device="cuda"))
    cache.check()
    assert int(cache.free_count) == cache.page_refs.shape[0]


if __name__ == "__main__":
    main()
