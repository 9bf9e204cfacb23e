"""Helpers of the tree-decoding tests: batches with drafted-token trees and
plain 64-bit implementations of the operators (numpy, from the formulas).

Tolerances, from the rounding the formulas allow (u = 2^-8 is bf16's unit
roundoff): an attention output is sum_j p_j v_j with p_j rounded to bf16 once
and the sum rounded to bf16 once, so |got - ref| <= u (sum_j p_j |v_j| + |ref|)
plus fp32 terms; lse is fp32 throughout: products of bf16 values are exact in
fp32 and 64 of them are summed, then 2^x and log2 to about 2^-21."""
import numpy as np
import torch

U = 2.0 ** -8
LSE_ABS = 1e-4


def bf(x):
    """float64 array -> (bf16 tensor on the CPU, its values as float64)."""
    t = torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16)
    return t, t.double().numpy()


def random_tree(n, rng, fan=4):
    """Parents of n nodes in topological order (-1: child of the context)."""
    return np.array([int(rng.integers(max(-1, i - fan), i)) if i else -1 for i in range(n)], np.int64)


def ancestors(parent):
    """[n, n] bool: node i sees node j (its ancestors and itself), and depths."""
    n = len(parent)
    sees = np.zeros((n, n), bool)
    depth = np.zeros(n, np.int64)
    for i in range(n):
        if parent[i] >= 0:
            sees[i] = sees[parent[i]]
            depth[i] = depth[parent[i]] + 1
        sees[i, i] = True
    return sees, depth


def pack_mask(sees_rows, words):
    """List of [n, n] bool per row -> int32 [T, words]."""
    out = []
    for sees in sees_rows:
        m = np.zeros((sees.shape[0], words), np.uint32)
        for j in range(sees.shape[1]):
            m[:, j // 32] |= sees[:, j].astype(np.uint32) << np.uint32(j % 32)
        out.append(m)
    return np.concatenate(out).view(np.int32) if out else np.zeros((0, words), np.int32)


class TreeBatch:
    """Rows with context lengths `ctx` and trees of `lens` nodes over a pool
    whose pages no row owns, and whose slots no row owns, hold NaN."""

    def __init__(self, ctx, lens, hq, hkv, seed, window=0, words=None, sees=None, scale=0.125, big=1.0):
        rng = np.random.default_rng(seed)
        self.ctx, self.lens = np.asarray(ctx, np.int64), np.asarray(lens, np.int64)
        self.hq, self.hkv, self.window, self.scale = hq, hkv, window, scale
        B = len(self.ctx)
        S = self.ctx + self.lens
        self.S = S
        self.qsl = np.concatenate([[0], np.cumsum(self.lens)])
        T = int(self.qsl[-1])
        trees = [ancestors(random_tree(int(n), rng)) for n in self.lens]
        self.sees = [t[0] for t in trees] if sees is None else sees
        self.words = words or max(1, (int(self.lens.max()) + 31) // 32)
        self.mask = pack_mask(self.sees, self.words)
        self.positions = np.concatenate([c + t[1] for c, t in zip(self.ctx, trees)]).astype(np.int64)
        last = (S + 15) // 16
        first = np.maximum(self.ctx - window + 1, 0) // 16 if window > 0 else np.zeros(B, np.int64)
        width = max(1, int(last.max()))
        P = int((last - first).clip(min=0).sum()) + 2
        ids = rng.permutation(P)
        self.bt = np.full((B, width), -1, np.int64)
        k = 0
        for r in range(B):
            for j in range(int(first[r]), int(last[r])):
                self.bt[r, j] = ids[k]
                k += 1
        kc = np.full((P, hkv, 16, 64), np.nan)
        vc = np.full((P, hkv, 16, 64), np.nan)
        for r in range(B):
            lo = max(0, int(self.ctx[r]) - window + 1) if window > 0 else 0
            pos = np.arange(lo, int(S[r]))
            kc[self.bt[r, pos // 16], :, pos % 16] = rng.standard_normal((len(pos), hkv, 64))
            vc[self.bt[r, pos // 16], :, pos % 16] = rng.standard_normal((len(pos), hkv, 64))
        (self.kt, self.k), (self.vt, self.v) = bf(kc), bf(vc)
        self.qt, self.q = bf(rng.standard_normal((T, hq, 64)) * big)

    def device(self):
        i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()  # noqa: E731
        return dict(q=self.qt.cuda(), kc=self.kt.cuda(), vc=self.vt.cuda(), bt=i32(self.bt), sl=i32(self.S),
                    qsl=i32(self.qsl), mask=i32(self.mask), pos=i32(self.positions))

    def reference(self, sinks=None):
        """(out, lse, sum_j p_j |v_j|) in 64 bits."""
        T = len(self.positions)
        out, mag = np.zeros((T, self.hq, 64)), np.zeros((T, self.hq, 64))
        lse = np.full((T, self.hq), -np.inf)
        g = self.hq // self.hkv
        for r in range(len(self.ctx)):
            C, n = int(self.ctx[r]), int(self.lens[r])
            for i in range(n):
                t = int(self.qsl[r]) + i
                p = min(max(int(self.positions[t]), C), C + n - 1)
                lo = max(0, p - self.window + 1) if self.window > 0 else 0
                keys = np.concatenate([np.arange(min(lo, C), C), C + np.nonzero(self.sees[r][i])[0]])
                if len(keys) == 0:
                    if sinks is not None:
                        lse[t] = sinks
                    continue
                page, slot = self.bt[r, keys // 16], keys % 16
                for h in range(self.hkv):
                    k, v = self.k[page, h, slot], self.v[page, h, slot]
                    hs = slice(h * g, (h + 1) * g)
                    s = self.scale * self.q[t, hs] @ k.T
                    m = s.max(1)
                    if sinks is not None:
                        m = np.maximum(m, sinks[hs])
                    w = np.exp(s - m[:, None])
                    z = w.sum(1) + (np.exp(sinks[hs] - m) if sinks is not None else 0)
                    out[t, hs] = w @ v / z[:, None]
                    mag[t, hs] = w @ np.abs(v) / z[:, None]
                    lse[t, hs] = m + np.log(z)
        return out, lse, mag


def assert_tree_close(out, lse, ref):
    ro, rl, mag = ref
    got = out.double().cpu().numpy()
    assert np.all(np.isfinite(got))
    bound = U * 1.01 * (mag + np.abs(ro)) + 1e-6
    worst = np.max(np.abs(got - ro) / bound) if got.size else 0.0
    assert worst <= 1.0, f"output off by {worst:.3f} of its bound"
    gl = lse.double().cpu().numpy()
    fin = np.isfinite(rl)
    assert np.array_equal(gl[~fin], rl[~fin])
    assert np.max(np.abs(gl[fin] - rl[fin]), initial=0.0) <= LSE_ABS
