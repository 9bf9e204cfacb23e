"""Per-head norm + rotation + KV append against a plain 64-bit implementation.

Tolerance: fp32 throughout and one rounding to bf16 (unit roundoff 2^-8): the
sum of 64 squares, the root, the reciprocal and four products are each within
a few 2^-24 relative, so |got - ref| <= 2^-8 |ref| + 2^-19 (|n_i| + |n_{i+32}|)."""
import ctypes

import numpy as np
import pytest
import torch

import workloads as W
from _tree import bf

gpu = pytest.mark.gpu


def _ref(x, w, eps, ang):
    """x [T, H, 64] -> rotated norm and the magnitude |n_i| + |n_{i+32}|."""
    m = (x * x).mean(-1, keepdims=True) + eps
    n = np.where(m > 0, x / np.sqrt(np.where(m > 0, m, 1)), 0) * w
    a, b = n[..., :32], n[..., 32:]
    c, s = ang[:, None, :32], ang[:, None, 32:]
    mag = np.abs(a) + np.abs(b)
    return np.concatenate([a * c - b * s, b * c + a * s], -1), np.concatenate([mag, mag], -1)


def _case(ctx, lens, hq, hkv, seed, packed, positions, size=1.0, gap=0):
    rng = np.random.default_rng(seed)
    ctx, lens = np.asarray(ctx), np.asarray(lens)
    S, T = ctx + lens, int(lens.sum())
    last = (S + 15) // 16
    P = int(last.sum()) + 2
    ids = rng.permutation(P)
    bt = np.full((len(S), max(1, int(last.max()))), -1, np.int64)
    k = 0
    for r in range(len(S)):
        bt[r, :last[r]] = ids[k:k + last[r]]
        k += int(last[r])
    width = (hq + 2 * hkv) * 64 + gap
    x, xv = bf(rng.standard_normal((T, width)) * size)
    cut = [(0, hq), (hq, hkv), (hq + hkv, hkv)]
    slot = np.concatenate([np.arange(c, s) for c, s in zip(ctx, S)]) if T else np.zeros(0, np.int64)
    row = np.repeat(np.arange(len(S)), lens)
    pos = rng.integers(0, 5000, T) if positions else slot
    x = x.cuda()
    parts = [x[:, a * 64:(a + h) * 64].unflatten(1, (h, 64)) for a, h in cut]
    if not packed:
        parts = [p.contiguous() for p in parts]
    vals = [xv[:, a * 64:(a + h) * 64].reshape(T, h, 64) for a, h in cut]
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()  # noqa: E731
    kc, vc = (torch.full((P, hkv, 16, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return dict(parts=parts, vals=vals, bt=bt, S=S, slot=slot, row=row, pos=pos, kc=kc, vc=vc, T=T,
                dbt=i32(bt), dsl=i32(S), dqsl=i32(np.concatenate([[0], np.cumsum(lens)])),
                dpos=i32(pos) if positions else None, status=torch.zeros(1, dtype=torch.int32, device="cuda"))


def _call(c, wq, wk, eps, tab, q_out=None):
    from paper_2608_22167_gb300 import mcpu

    q, k, v = c["parts"]
    q_out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda") if q_out is None else q_out
    f32 = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda()  # noqa: E731
    mcpu.mcpu_norm_rope_kv_append(q, k, v, f32(wq), f32(wk), eps, c["dpos"], tab, q_out, c["kc"], c["vc"], c["dbt"],
                                  c["dsl"], c["dqsl"], c["status"])
    return q_out


def _compare(c, q_out, wq, wk, eps, tab):
    ang = tab.double().cpu().numpy()[c["pos"]]
    page, slot = c["bt"][c["row"], c["slot"] // 16], c["slot"] % 16
    kc, vc = c["kc"].double().cpu().numpy(), c["vc"].double().cpu().numpy()
    eps = float(np.float32(eps))
    for got, x, w in ((q_out.double().cpu().numpy(), c["vals"][0], wq), (kc[page, :, slot], c["vals"][1], wk)):
        ref, mag = _ref(x, np.asarray(w, np.float32).astype(np.float64), eps, ang)
        assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -19 * mag)
    assert np.array_equal(vc[page, :, slot], c["vals"][2])
    untouched = np.ones(kc.shape[:1] + (16,), bool)
    untouched[page, slot] = False
    assert np.all(kc.transpose(0, 2, 1, 3)[untouched] == 7.0) and np.all(vc.transpose(0, 2, 1, 3)[untouched] == 7.0)
    assert int(c["status"].item()) == 0


@gpu
@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("positions", [True, False])
@pytest.mark.parametrize("hq,hkv", [(64, 8), (8, 2), (16, 2), (3, 3), (1, 1)])
def test_matches_the_formula(hq, hkv, packed, positions):
    rng = np.random.default_rng(hq)
    tab = torch.from_numpy(W.rope_table(5000)).cuda()
    wq, wk = 1 + 0.3 * rng.standard_normal(64), 1 + 0.3 * rng.standard_normal(64)
    for ctx, lens in (([5], [1]), ([0, 15, 16, 40], [1, 1, 1, 1]), ([0, 7, 130, 0, 33], [20, 1, 64, 0, 117]),
                      (rng.integers(0, 100, 70), rng.integers(0, 6, 70))):
        c = _case(ctx, lens, hq, hkv, 1, packed, positions, size=2.0, gap=8)
        _compare(c, _call(c, wq, wk, 1e-6, tab), wq, wk, 1e-6, tab)


@gpu
@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("hq,hkv", [(64, 8), (8, 2), (32, 8), (1, 1), (5, 5), (96, 12), (128, 64)])
def test_many_tokens(hq, hkv, packed):
    # enough tokens for every form of the kernel on any SM count of this GPU, odd totals, empty rows
    rng = np.random.default_rng(hq + 1)
    tab = torch.from_numpy(W.rope_table(5000)).cuda()
    wq, wk = 1 + 0.3 * rng.standard_normal(64), 1 + 0.3 * rng.standard_normal(64)
    for total in (700, 2431, 2433, 4999):
        lens = rng.multinomial(total, np.ones(37) / 37)
        lens[5] += lens[6]
        lens[6] = 0
        c = _case(rng.integers(0, 200, 37), lens, hq, hkv, total, packed, total % 2 == 0, gap=16)
        _compare(c, _call(c, wq, wk, 1e-6, tab), wq, wk, 1e-6, tab)


@gpu
def test_many_tokens_with_errors():
    from paper_2608_22167_gb300 import mcpu

    tab = torch.from_numpy(W.rope_table(900)).cuda()
    w = np.ones(64)
    c = _case([0, 500, 30], [3000, 700, 900], 8, 2, 9, True, False)  # positions from 900 on lie past the table
    c["dbt"][2, 3] = -1  # tokens at slots 48 .. 63 of row 2 have no page
    out = _call(c, w, w, 1e-6, tab).float().cpu()
    bad = torch.zeros(4600, dtype=torch.bool)
    bad[900:3000] = True
    bad[3400:3700] = True
    bad[4570:] = True
    assert torch.isnan(out[bad]).all() and torch.isfinite(out[~bad]).all()
    assert int(c["status"].item()) == mcpu.STATUS_BAD_LENGTHS | mcpu.STATUS_BAD_PAGE
    slot = np.where((c["row"] == 2) & (c["slot"] // 16 == 3), -1, c["slot"])
    keep = (slot >= 0) & ~bad.numpy()
    page = c["bt"][c["row"], c["slot"] // 16]
    vc = c["vc"].double().cpu().numpy()
    assert np.array_equal(vc[page[keep], :, c["slot"][keep] % 16], c["vals"][2][keep])
    assert np.all(vc[page[~keep], :, c["slot"][~keep] % 16] == 7)


@gpu
@pytest.mark.parametrize("size", [1e-8, 1e-3, 1e8])
def test_small_and_large_values(size):
    tab = torch.from_numpy(W.rope_table(600)).cuda()
    w = np.linspace(-2, 2, 64)
    for eps in (0.0, 1e-6):
        c = _case([3, 500], [10, 1], 16, 2, 2, True, False, size=size)
        _compare(c, _call(c, w, w, eps, tab), w, w, eps, tab)


@gpu
def test_tables_and_weights_at_any_float():
    big = torch.zeros(600 * 64 + 1, device="cuda")
    big[1:] = torch.from_numpy(W.rope_table(600)).cuda().flatten()
    tab = big[1:].view(600, 64)  # 4-byte aligned only
    assert tab.data_ptr() % 16 == 4
    w = np.linspace(-2, 2, 64)
    c = _case([3, 500], [10, 1], 16, 2, 2, True, False)
    _compare(c, _call(c, w, w, 1e-6, tab), w, w, 1e-6, tab)


@gpu
def test_zero_rows_and_in_place():
    tab = torch.from_numpy(W.rope_table(600)).cuda()
    w = np.ones(64)
    c = _case([3, 500], [10, 1], 16, 2, 3, False, False)
    c["parts"][0][4].zero_()
    c["vals"][0][4] = 0
    q = c["parts"][0]
    out = _call(c, w, w, 0.0, tab, q_out=q)  # in place, eps 0: a zero row stays zero
    assert out is q
    _compare(c, out, w, w, 0.0, tab)


@gpu
def test_device_errors_leave_the_token_alone():
    from paper_2608_22167_gb300 import mcpu

    tab = torch.from_numpy(W.rope_table(100)).cuda()
    w = np.ones(64)
    c = _case([0, 0, 0], [2, 3, 2], 8, 2, 4, True, True)
    pos = torch.tensor([1, 2, 100, -1, 5, 6, 7], dtype=torch.int32, device="cuda")
    c["dpos"] = pos
    c["dbt"][2, 0] = 1 << 20  # row 2's page lies outside the pool
    out = _call(c, w, w, 1e-6, tab).float().cpu()
    assert torch.isnan(out[2:4]).all() and torch.isfinite(out[[0, 1, 4, 5, 6]]).all()
    bits = int(c["status"].item())
    assert bits == mcpu.STATUS_BAD_LENGTHS | mcpu.STATUS_BAD_PAGE
    kc = c["kc"].float().cpu()
    assert torch.all(kc[c["bt"][1, 0], :, :2] == 7) and torch.all(kc[c["bt"][2, 0]] == 7)
    assert torch.all(kc[c["bt"][1, 0], :, 2] != 7) and torch.all(kc[c["bt"][0, 0], :, :2] != 7)


def test_host_checks():
    from paper_2608_22167_gb300 import mcpu

    f = mcpu._lib.mcpu_norm_rope_kv_append
    P = 1 << 20
    ok = dict(q=P, qs=512, k=P, ks=128, v=P, vs=128, wq=P, wk=P, eps=1e-6, pos=None, tab=P, mp=10, out=P + 4096, kc=P,
              vc=P, bt=P, sl=P, qsl=P, dims=mcpu.Dims(4, 9, 19, 34, 8, 2, 64, 16), st=P)

    def call(**kw):
        a = dict(ok, **kw)
        return f(a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["wq"], a["wk"], a["eps"], a["pos"], a["tab"],
                 a["mp"], a["out"], a["kc"], a["vc"], a["bt"], a["sl"], a["qsl"], ctypes.byref(a["dims"]), a["st"], None)

    for name in ("q", "k", "v", "wq", "wk", "tab", "out", "kc", "vc", "bt", "sl", "qsl", "st"):
        assert call(**{name: None}) == 1, name
    for name in ("q", "k", "v", "out", "kc", "vc"):
        assert call(**{name: P + 8}) == 1, name
    assert call(pos=P + 2) == 1 and call(mp=0) == 1
    for eps in (-1e-6, float("nan"), float("inf")):
        assert call(eps=eps) == 1
    assert call(qs=504) == 1 and call(qs=516) == 1 and call(ks=120) == 1 and call(vs=132) == 1
    assert call(out=P, qs=1024) == 1  # in place needs a dense q
    assert call(dims=mcpu.Dims(4, 9, 19, 34, 8, 2, 32, 16)) == 2
    assert call(dims=mcpu.Dims(0, 0, 19, 34, 8, 2, 64, 16)) == 0


def test_binding_checks():
    from paper_2608_22167_gb300 import mcpu

    z = torch.zeros
    q, k = z(4, 8, 64, dtype=torch.bfloat16), z(4, 2, 64, dtype=torch.bfloat16)
    kc = z(3, 2, 16, 64, dtype=torch.bfloat16)
    i = z(1, dtype=torch.int32)
    args = dict(q=q, k_new=k, v_new=k, q_weight=z(64), k_weight=z(64), eps=1e-6, positions=None, cos_sin=z(9, 64),
                q_out=q.clone(), k_cache=kc, v_cache=kc, block_table=z(1, 3, dtype=torch.int32), seq_lens=i,
                query_start_loc=i, status_word=i, stream=object())
    for bad in (dict(cos_sin=z(9, 32)), dict(q_weight=z(32)), dict(k_weight=z(64, dtype=torch.bfloat16)),
                dict(q_out=q.float()), dict(positions=z(3, dtype=torch.int32)), dict(k_new=k[:3]),
                dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)), dict(positions=z(4, dtype=torch.int64))):
        with pytest.raises(ValueError):
            mcpu.mcpu_norm_rope_kv_append(**dict(args, **bad))


@gpu
@pytest.mark.parametrize("tokens", [11, 3000])
def test_a_nan_reaches_all_of_its_head_and_nothing_else(tokens):
    tab = torch.from_numpy(W.rope_table(5000)).cuda()
    w = np.ones(64)
    c = _case([3, 500], [tokens - 1, 1], 16, 2, 3, False, False)
    good = _call(c, w, w, 1e-6, tab).clone()
    kept = c["kc"].clone(), c["vc"].clone()
    for part, token, head, dim in ((0, 4, 2, 5), (0, tokens - 1, 15, 63), (1, 4, 1, 40)):
        c["parts"][part][token, head, dim] = float("nan")
    out = _call(c, w, w, 1e-6, tab)
    bad = torch.zeros(tokens, 16, dtype=torch.bool)
    bad[4, 2] = bad[tokens - 1, 15] = True
    assert torch.isnan(out.cpu()[bad]).all() and torch.equal(out.cpu()[~bad], good.cpu()[~bad])
    page, slot = c["bt"][0, 7 // 16], 7
    assert torch.isnan(c["kc"][page, 1, slot]).all()
    c["kc"][page, 1, slot] = kept[0][page, 1, slot]
    assert torch.equal(c["kc"], kept[0]) and torch.equal(c["vc"], kept[1])
    assert int(c["status"].item()) == 0
