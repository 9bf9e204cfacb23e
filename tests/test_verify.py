"""mcpu_verify_tree against a plain walk in 64 bits, and what it refuses."""
import numpy as np
import pytest
import torch

from _tree import random_tree
from _verify import reference

gpu = pytest.mark.gpu


def _case(lens, vocab, seed, fp32=False, draft=False, heats=(0.8,), most=None, spread=2.0):
    """Random trees whose children's tokens are often the likeliest of their node."""
    rng = np.random.default_rng(seed)
    qsl = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    T = int(qsl[-1])
    dtype = torch.float32 if fp32 else torch.bfloat16
    x = torch.from_numpy(rng.standard_normal((T, vocab)) * spread)
    y = (x + torch.from_numpy(rng.standard_normal((T, vocab)) * 0.7)).to(dtype)
    x = x.to(dtype)
    logits, drafts = x.double().numpy(), y.double().numpy()
    parents = np.concatenate([random_tree(int(n), rng) for n in lens]) if T else np.zeros(0, np.int64)
    parents = np.where(parents < 0, -1, parents)
    tokens = rng.integers(0, vocab, T)
    for r, n in enumerate(lens):
        born = {}
        for i in range(1, int(n)):
            t, up = int(qsl[r]) + i, int(parents[qsl[r] + i])
            if up < 0:
                continue
            k = born[up] = born.get(up, -1) + 1
            src = drafts if draft else logits
            if k < vocab and rng.random() < 0.8:
                tokens[t] = np.argsort(-src[qsl[r] + up], kind="stable")[k]
    heat = np.array([heats[r % len(heats)] for r in range(len(lens))], np.float32)
    u = rng.random(T).astype(np.float32)
    noise = np.maximum(rng.exponential(size=(len(lens), vocab)), 1e-6).astype(np.float32)
    return dict(x=x, y=y if draft else None, logits=logits, draft=drafts if draft else None, tokens=tokens,
                parents=parents, qsl=qsl, heat=heat, u=u, noise=noise, most=most or max(1, int(max(lens, default=1))))


def _call(c, logits=None, draft=None, noise=None, no_heat=False, status=None):
    from paper_2608_22167_gb300 import mcpu

    dev = "cuda"
    i32 = lambda a: torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device=dev)  # noqa: E731
    f32 = lambda a: torch.as_tensor(np.ascontiguousarray(a), dtype=torch.float32, device=dev)  # noqa: E731
    rows, most = len(c["qsl"]) - 1, c["most"]
    path = torch.full((rows, most), 77, dtype=torch.int32, device=dev)
    length, following = (torch.full((rows,), 77, dtype=torch.int32, device=dev) for _ in range(2))
    logp = torch.full((rows, most), 77.0, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev) if status is None else status
    logits = c["x"].to(dev) if logits is None else logits
    draft = (c["y"].to(dev) if c["y"] is not None else None) if draft is None else draft
    noise = f32(c["noise"]) if noise is None else noise
    mcpu.mcpu_verify_tree(logits, i32(c["tokens"]), i32(c["parents"]), i32(c["qsl"]),
                          None if no_heat else f32(c["heat"]), None if no_heat else f32(c["u"]),
                          None if no_heat else noise, path, length, following, logp, status, draft_logits=draft)
    return path.cpu().numpy(), length.cpu().numpy(), following.cpu().numpy(), logp.double().cpu().numpy(), int(status)


def _check(got, c, rows=None):
    """Whole numbers equal. A log-probability is a difference and the log of a sum: each term 2^t of the sum is off by
    (|t| + 3) 2^-24 relative, less than 40 of them where it weighs anything, the sum of vocab / 256 terms a thread by as
    many 2^-24, and the result is rounded once."""
    want = reference(c)
    assert want[4] > 1e-4, "inputs with a decision this close to its border say nothing"
    rows = slice(None) if rows is None else rows
    for g, w in zip(got[:3], want[:3]):
        assert np.array_equal(g[rows], w[rows])
    bound = 2.0 ** -24 * (40 + c["logits"].shape[1] / 256) + 2.0 ** -24 * np.abs(want[3])
    assert np.all(np.abs(got[3] - want[3])[rows] <= bound[rows])


LENS = [1, 2, 0, 5, 17, 40, 3, 9]


@gpu
@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("draft", [False, True])
@pytest.mark.parametrize("vocab", [1, 2, 7, 33, 257, 1000, 4099, 32000])
def test_matches_the_plain_walk(vocab, draft, fp32):
    c = _case(LENS, vocab, seed=11 + vocab, fp32=fp32, draft=draft, heats=(0.8, 0.0, 1.3))
    got = _call(c)
    assert got[4] == 0
    _check(got, c)


@gpu
@pytest.mark.parametrize("rows", [1, 3, 20, 100, 300])
@pytest.mark.parametrize("draft", [False, True])
def test_any_number_of_rows(rows, draft):
    # few rows are walked by several blocks each, many by one
    rng = np.random.default_rng(rows)
    c = _case(rng.integers(1, 7, rows), 9001, seed=rows, draft=draft, heats=(1.0, 0.5))
    _check(_call(c), c)


@gpu
@pytest.mark.parametrize("vocab", [131072, 200019])
def test_large_vocabularies(vocab):
    c = _case([4, 6, 1], vocab, seed=vocab, draft=True, spread=3.0)
    _check(_call(c), c)


@gpu
def test_strided_and_unaligned_rows():
    c = _case(LENS, 1003, seed=5, draft=True)
    for off, pad in ((0, 1), (1, 0), (3, 8), (5, 2)):
        def place(t, dtype):
            wide = torch.full((t.shape[0], t.shape[1] + pad + off + 8), float("nan"), dtype=dtype, device="cuda")
            wide[:, off:off + t.shape[1]] = t.to("cuda")
            return wide[:, off:off + t.shape[1]]

        got = _call(c, place(c["x"], torch.bfloat16), place(c["y"], torch.bfloat16),
                    place(torch.from_numpy(c["noise"]), torch.float32))
        _check(got, c)


@gpu
def test_paths_end_at_max_accept():
    c = _case([12] * 6, 50, seed=3, heats=(0.0, 0.7), most=3)
    c["parents"] = np.tile(np.arange(-1, 11), 6)
    got = _call(c)
    _check(got, c)
    c["most"] = 1  # no child is tried: plain sampling after the last token
    got = _call(c)
    _check(got, c)
    assert np.all(got[1] == 1)


@gpu
@pytest.mark.parametrize("draft", [False, True])
def test_repeated_padded_and_unreachable_nodes(draft):
    c = _case([30] * 8, 64, seed=8, draft=draft)
    rng = np.random.default_rng(9)
    c["tokens"] = rng.integers(0, 4, 240)  # siblings with the same token
    c["tokens"][rng.random(240) < 0.2] = -1
    c["tokens"][rng.random(240) < 0.1] = 64
    far = rng.random(240) < 0.1
    c["parents"] = np.where(far, rng.integers(-5, 300, 240), c["parents"])
    c["x"][:, :4] += 3
    c["logits"] = c["x"].double().numpy()
    _check(_call(c), c)


@gpu
def test_masked_tokens():
    for draft in (False, True):
        c = _case(LENS, 300, seed=21, draft=draft, heats=(0.0, 1.0))
        hide = torch.from_numpy(np.random.default_rng(2).random(c["x"].shape) < 0.9)
        hide[:, 7] = False
        c["x"][hide] = -torch.inf
        c["logits"] = c["x"].double().numpy()
        with np.errstate(divide="ignore", invalid="ignore"):
            got, want = _call(c), reference(c)
        assert got[4] == 0 and want[4] > 1e-4
        for g, w in zip(got[:3], want[:3]):
            assert np.array_equal(g, w)
        # masks of the type's lowest value weigh nothing either, unless there is nothing else
        low = _call(dict(c, x=torch.where(hide, torch.finfo(torch.bfloat16).min, c["x"])))
        for g, w in zip(low[:3], want[:3]):
            assert np.array_equal(g, w)


@gpu
def test_rows_of_the_lowest_value_are_uniform():
    c = _case([1] * 3, 10, seed=1)
    c["x"][:] = torch.finfo(torch.bfloat16).min
    c["logits"] = c["x"].double().numpy()
    _check(_call(c), c)


@gpu
def test_ties_go_to_the_lowest_token():
    c = _case([1, 1, 2], 5000, seed=4, heats=(0.0, 1.0, 0.0))
    c["x"][:] = 0
    c["x"][:, 1234] = c["x"][:, 4321] = c["x"][:, 40] = 5
    c["logits"], c["noise"][:] = c["x"].double().numpy(), 1
    c["tokens"][:], c["parents"][:] = 40, [-1, -1, -1, 0]
    got = _call(c)
    assert got[2].tolist() == [40, 40, 40] and got[1].tolist() == [1, 1, 2]
    c["tokens"][:] = 4321
    assert _call(c)[1].tolist() == [1, 1, 1]


@gpu
def test_without_temperature_all_rows_are_greedy():
    c = _case(LENS, 500, seed=6, heats=(0.0,))
    _check(_call(c, no_heat=True), c)


@gpu
@pytest.mark.parametrize("what", ["nan", "inf", "nothing", "draft_nan", "heat_nan", "heat_low", "heat_negative"])
def test_rows_without_a_distribution_are_reported(what):
    c = _case([3, 3, 3], 77, seed=12, draft=True)
    c["heat"][1] = 1.0
    good = _call(c)
    if what == "nan":
        c["x"][3, 70] = torch.nan
    elif what == "inf":
        c["x"][3, 0] = torch.inf
    elif what == "nothing":
        c["x"][3] = -torch.inf
    elif what == "draft_nan":
        c["y"][3, 76] = torch.nan
    else:
        c["heat"][1] = dict(heat_nan=np.nan, heat_low=1e-30, heat_negative=-1.0)[what]
    got = _call(c)
    assert got[4] == 64
    assert got[0][1].tolist() == [0, -1, -1] and got[1][1] == 1 and got[2][1] == -1 and np.isnan(got[3][1, 0])
    for g, w in zip(got[:4], good[:4]):
        assert np.array_equal(g[[0, 2]], w[[0, 2]])


@gpu
def test_bad_rows_are_reported_and_skipped():
    c = _case([2, 257, 4], 40, seed=30)
    got = _call(c)
    assert got[4] == 32 and got[1][1] == 0 and got[2][1] == -1 and np.all(got[0][1] == -1) and not got[3][1].any()
    assert got[1][0] >= 1 and got[1][2] >= 1
    c = _case([2, 256, 4], 40, seed=31)
    _check(_call(c), c)
    for qsl in ([0, 3, 2, 9], [0, 2, 5, 8], [1, 2, 5, 9]):
        c = _case([2, 3, 4], 40, seed=30)
        c["qsl"] = np.array(qsl)
        got = _call(c)
        assert got[4] == 2


@gpu
def test_offsets_past_32_bits():
    c = _case([2, 1], 1000, seed=13, draft=True)
    buf = torch.empty(2 * (2 ** 31 + 5) + 1000, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((3, 1000), (2 ** 31 + 5, 1))
    far.copy_(c["x"])
    _check(_call(c, logits=far), c)
    far.copy_(c["y"])
    _check(_call(c, draft=far), c)
    noise = torch.empty(2 ** 31 + 1008, device="cuda").as_strided((2, 1000), (2 ** 31 + 8, 1))
    noise.copy_(torch.from_numpy(c["noise"]))
    _check(_call(c, noise=noise), c)


@gpu
@pytest.mark.parametrize("draft", [False, True])
def test_emitted_tokens_follow_the_target(draft):
    """The first two emitted tokens of many rows with the same logits have the target's joint distribution, whatever
    the draft proposes. A count of n p tokens has the deviation sqrt(n p (1 - p)): five of them hold with 1 - 6e-7."""
    from paper_2608_22167_gb300 import mcpu

    V, rows, rounds, heat = 8, 2048, 40, 0.9
    g = torch.Generator(device="cuda")
    g.manual_seed(5 + draft)
    x = torch.randn(1 + V, V, generator=g, device="cuda") * 1.2  # after the root, and after each first token
    y = torch.randn(1 + V, V, generator=g, device="cuda") * 1.2
    q = (y / heat).softmax(1)
    i32 = dict(dtype=torch.int32, device="cuda")
    seen = torch.zeros(V, V, device="cuda", dtype=torch.float64)
    nodes = 1 + 3 + 3  # the root, three drafts of the first token, three below the first of them
    parents = torch.tensor([-1, 0, 0, 0, 1, 1, 1], **i32).repeat(rows)
    qsl = torch.arange(0, rows * nodes + 1, nodes, **i32)
    for _ in range(rounds):
        if draft:
            first = torch.multinomial(q[0].expand(rows, V), 3, True, generator=g)
            second = torch.multinomial(q[1 + first[:, 0]], 3, True, generator=g)
        else:
            first, second = torch.tensor([5, 1, 2], device="cuda").expand(rows, 3), torch.tensor([0, 5, 7], device="cuda").expand(rows, 3)
        root = torch.zeros(rows, 1, dtype=torch.int64, device="cuda")
        tokens = torch.cat([root, first, second], 1)
        at = torch.cat([root, 1 + first, 1 + second], 1)  # rows of x and y that each node's logits are
        path, n, nxt = torch.empty(rows, 3, **i32), torch.empty(rows, **i32), torch.empty(rows, **i32)
        status = torch.zeros(1, **i32)
        mcpu.mcpu_verify_tree(x[at].view(-1, V), tokens.int().view(-1), parents, qsl,
                              torch.full((rows,), heat, device="cuda"),
                              torch.rand(rows * nodes, generator=g, device="cuda"),
                              torch.empty(rows, V, device="cuda").exponential_(generator=g).clamp_(min=1e-9), path, n,
                              nxt, None, status, draft_logits=y[at].view(-1, V) if draft else None)
        assert int(status) == 0
        emitted = torch.where(torch.arange(2, device="cuda") < (n - 1)[:, None],
                              tokens.gather(1, path[:, 1:].long().clamp(min=0)), nxt.long()[:, None])
        # the second token, where the round ended with the first: drawn plainly
        plain = torch.multinomial((x[1 + emitted[:, 0]] / heat).softmax(1), 1, generator=g)[:, 0]
        second = torch.where(n >= 2, emitted[:, 1], plain)
        seen.view(-1).index_add_(0, emitted[:, 0] * V + second, torch.ones(rows, device="cuda", dtype=torch.float64))
    total = rows * rounds
    p = (x.double() / heat).softmax(1)
    want = p[0][:, None] * p[1:]
    assert torch.all((seen - total * want).abs() <= 5 * (total * want * (1 - want)).sqrt() + 1)


@gpu
def test_replays_follow_their_inputs_and_other_streams_work():
    from paper_2608_22167_gb300 import mcpu

    c, d = _case(LENS, 900, seed=40, draft=True), _case(LENS, 900, seed=41, draft=True)
    dev = lambda a, t: torch.as_tensor(np.ascontiguousarray(a), dtype=t, device="cuda")  # noqa: E731
    keys = dict(tokens=torch.int32, parents=torch.int32, heat=torch.float32, u=torch.float32, noise=torch.float32)
    t = {k: dev(c[k], v) for k, v in keys.items()}
    x, y, qsl = c["x"].cuda(), c["y"].cuda(), dev(c["qsl"], torch.int32)
    rows, most = len(LENS), c["most"]
    path, n, nxt = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((rows, most), (rows,), (rows,)))
    logp, status = torch.empty(rows, most, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(stream=None):
        mcpu.mcpu_verify_tree(x, t["tokens"], t["parents"], qsl, t["heat"], t["u"], t["noise"], path, n, nxt, logp,
                              status, draft_logits=y, stream=stream)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    run(side)
    side.synchronize()
    _check((path.cpu().numpy(), n.cpu().numpy(), nxt.cpu().numpy(), logp.double().cpu().numpy()), c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    x.copy_(d["x"])
    y.copy_(d["y"])
    for k, v in keys.items():
        t[k].copy_(dev(d[k], v))
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        _check((path.cpu().numpy(), n.cpu().numpy(), nxt.cpu().numpy(), logp.double().cpu().numpy()), d)


def _near(case, got):
    """The walks of draws that lie next to a border: paths and their lengths as in 64 bits."""
    want = reference(case)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


@gpu
@pytest.mark.parametrize("vocab,first", [(40, 1), (40, 33), (4099, 1), (4099, 33), (60000, 1)])
@pytest.mark.parametrize("fp32", [False, True])
def test_siblings_of_tokens_that_take_almost_all(vocab, first, fp32):
    """Children left after the likeliest tokens were rejected: what remains, down to 1e-6 of the probability, is as
    good as the weights themselves. With d = (max - l) / T a weight is off by 2^-22 (its exponential) and 3 2^-24 d
    (three roundings of its exponent), relatively; here d < 30. Two of them in a quotient: 2 (2^-22 + 3 2^-24 30) =
    1.12e-5, and 40 2^-24 = 2.4e-6 for the sums. What is left may be a difference down to a quarter of the whole, where
    the roundings of the whole (12 2^-24 beside its likeliest terms, 2^-22 of what was taken off) count four times:
    3.8e-6. Draws 2e-5 on either side of a border are decided as in 64 bits."""
    rng = np.random.default_rng(vocab + first)
    cases = []
    for leaders in (1, 2):
        for rest in (0.3, 0.1, 1e-2, 1e-3, 1e-4, 1e-5, 1e-6):
            x = rng.standard_normal(vocab)
            top = rng.choice(vocab, leaders + 2, replace=False)
            x[top[:leaders]] = -np.inf
            height = np.log(np.exp(x).sum() * (1 - rest) / rest / leaders)
            x[top[:leaders]] = height - 0.01 * np.arange(leaders)
            x = torch.from_numpy(x).to(torch.float32 if fp32 else torch.bfloat16)
            p = np.exp(x.double().numpy() - x.double().numpy().max())
            p[top[:leaders]] = 0
            for kid in range(2):  # the border of the first sibling, or of the second once that is rejected
                level = p[top[leaders + kid]] / p.sum()
                p[top[leaders]] = 0
                for side in (-2e-5, 2e-5):
                    u = [1 - 2.0 ** -24] * (leaders + kid) + [level * (1 + side)]
                    cases.append((x, top[: leaders + kid + 1], u))
    # the children as nodes from `first` on, padding between
    nodes = first + 4
    B = len(cases)
    tokens, parents = np.full((B, nodes), -1), np.zeros((B, nodes), np.int64)
    parents[:, 0], u = -1, np.full((B, nodes), 0.5, np.float32)
    logits = torch.zeros(B, nodes, vocab, dtype=cases[0][0].dtype)
    for r, (x, kids, draws) in enumerate(cases):
        logits[r, 0] = x
        tokens[r, 0] = 0
        tokens[r, first : first + len(kids)] = kids
        u[r, first : first + len(kids)] = draws
    logits = logits.view(B * nodes, vocab)
    noise = np.maximum(rng.exponential(size=(B, vocab)), 1e-6).astype(np.float32)
    c = dict(x=logits, y=None, logits=logits.double().numpy(), draft=None, tokens=tokens.ravel(), parents=parents.ravel(),
             qsl=np.arange(0, B * nodes + 1, nodes), heat=np.ones(B, np.float32), u=u.ravel(), noise=noise, most=3)
    for lo in range(0, B, 8 if vocab > 10000 else B):  # few rows: several blocks each
        hi = min(B, lo + (8 if vocab > 10000 else B))
        part = dict(c, x=logits[lo * nodes : hi * nodes], logits=c["logits"][lo * nodes : hi * nodes],
                    tokens=c["tokens"][lo * nodes : hi * nodes], parents=c["parents"][lo * nodes : hi * nodes],
                    qsl=c["qsl"][: hi - lo + 1], heat=c["heat"][lo:hi], u=c["u"][lo * nodes : hi * nodes],
                    noise=noise[lo:hi])
        got = _call(part)
        assert got[4] == 0
        _near(part, got)


@gpu
@pytest.mark.parametrize("fp32", [False, True])
def test_drafts_close_to_their_target(fp32):
    """p - q of nearly equal p and q, both good to e = 2^-22 + 3 2^-24 d (see above; d < 8) and twice that with their
    sums: off by 4 e p, and the residual's mass by as much of the whole. Draws twice that far from a border."""
    vocab, rng = 2000, np.random.default_rng(23)
    dtype = torch.float32 if fp32 else torch.bfloat16
    e = 2.0 ** -22 + 24 * 2.0 ** -24
    rows = []
    for noise in (0.1, 0.01, 1e-3):
        x = torch.from_numpy(rng.standard_normal(vocab)).to(dtype)
        y = (x.double() + torch.from_numpy(rng.standard_normal(vocab) * noise)).to(dtype)
        p, q = (torch.softmax(t.double(), 0).numpy() for t in (x, y))
        r = np.maximum(p - q, 0)
        m = r.sum()
        if m == 0:
            continue
        kid = int(np.argmax(r / p * (r < m * q)))  # rejected at times, with as much of p left as there is
        level = r[kid] / m / q[kid]
        off = 8 * e * (p[kid] / r[kid] + 1 / m)
        lost = int(np.argmin(p / q))  # rejected by any draw above p / q
        for side in (-off, off):
            if 0 < level * (1 + side) < 1:
                rows.append((x, y, [lost, kid], [1 - 2.0 ** -24, level * (1 + side)]))
    assert len(rows) >= 4
    B = len(rows)
    x = torch.stack([t for r in rows for t in (r[0], r[0], r[0])])
    y = torch.stack([t for r in rows for t in (r[1], r[1], r[1])])
    c = dict(x=x, y=y, logits=x.double().numpy(), draft=y.double().numpy(), tokens=np.array([[0] + r[2] for r in rows]).ravel(),
             parents=np.tile([-1, 0, 0], B), qsl=np.arange(0, 3 * B + 1, 3), heat=np.ones(B, np.float32),
             u=np.array([[0.5] + r[3] for r in rows], np.float32).ravel(),
             noise=np.maximum(rng.exponential(size=(B, vocab)), 1e-6).astype(np.float32), most=2)
    _near(c, _call(c))


@gpu
@pytest.mark.parametrize("rows", [1, 3, 400])
@pytest.mark.parametrize("heat", [0.0, 1.0])
def test_rows_with_nothing_but_the_lowest_value_of_32_bits(rows, heat):
    vocab = 40000
    c = _case([1] * rows, vocab, seed=24, fp32=True, heats=(heat,))
    c["x"][:] = -torch.inf
    for r in range(rows):
        at = [39000 - 61 * r, 39990 - r, 39999]
        c["x"][r, at] = torch.finfo(torch.float32).min
    c["logits"] = c["x"].double().numpy()
    got, want = _call(c), reference(c)
    assert got[4] == 0
    for g, w in zip(got[:3], want[:3]):
        assert np.array_equal(g, w)
    assert np.all(np.abs(got[3] - want[3]) <= 2.0 ** -22)


@gpu
@pytest.mark.parametrize("fp32", [False, True])
def test_greedy_rows_take_what_the_host_takes(fp32):
    from paper_2608_22167_gb300.tree_decode import accept_greedy

    c = _case(np.arange(1, 65), 500, seed=25, fp32=fp32, heats=(0.0,), spread=0.7)
    c["parents"] = np.concatenate([np.maximum(random_tree(n, np.random.default_rng(n)), np.where(np.arange(n), 0, -1))
                                   for n in range(1, 65)])
    path, length, following, _, status = _call(c)
    assert status == 0 and length.max() > 2
    for r, (a, b) in enumerate(zip(c["qsl"], c["qsl"][1:])):
        want, token = accept_greedy(c["parents"][a:b].tolist(), c["tokens"][a:b].tolist(), c["logits"][a:b].argmax(1))
        assert path[r, : length[r]].tolist() == want and following[r] == token


def _args():
    """Valid arguments (CPU tensors: nothing is launched)."""
    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t)  # noqa: E731
    f32 = torch.float32
    return dict(logits=z(6, 30, t=torch.bfloat16), tokens=z(6), parents=z(6), query_start_loc=z(4),
                temperature=z(3, t=f32), uniforms=z(6, t=f32), exponentials=z(3, 30, t=f32), accept_path=z(3, 4),
                accept_len=z(3), next_token=z(3), logprobs=z(3, 4, t=f32), status_word=z(1),
                draft_logits=z(6, 30, t=torch.bfloat16), stream=None)


def test_binding_refuses_what_it_would_misread():
    from paper_2608_22167_gb300 import mcpu

    args = _args()
    with pytest.raises(ValueError, match="CUDA device"):  # the arguments as they are get as far as this
        mcpu.mcpu_verify_tree(**args)
    for key, x in args.items():
        if not torch.is_tensor(x):
            continue
        wrong = [x.double() if x.is_floating_point() else x.long()]
        if x.shape[-1] > 1:
            wrong.append(torch.stack([x, x], -1)[..., 0])
        if key != "status_word":
            wrong.append(x[:-1])
        if x.dim() == 2 and key not in ("accept_path",):
            wrong.append(x[:, :-1])
        for bad in wrong:
            with pytest.raises(ValueError, match="^(?!.*CUDA device)"):
                mcpu.mcpu_verify_tree(**dict(args, **{key: bad}))
    for bad in (dict(uniforms=None), dict(exponentials=None), dict(accept_path=torch.zeros(3, 0, dtype=torch.int32)),
                dict(logits=torch.zeros(1, 30, dtype=torch.bfloat16).expand(6, 30)),
                dict(draft_logits=torch.zeros(6, 30))):
        with pytest.raises(ValueError, match="^(?!.*CUDA device)"):
            mcpu.mcpu_verify_tree(**dict(args, **bad))


def test_batches_without_nodes_have_no_rows_to_be_dense():
    """An empty tensor's strides say nothing (of an array without rows they may be anything)."""
    from paper_2608_22167_gb300 import mcpu

    args = _args()
    none = torch.zeros(0, dtype=torch.int32)
    logits = torch.zeros(0, 30, dtype=torch.bfloat16).as_strided((0, 30), (1, 2))
    args.update(logits=logits, draft_logits=logits, tokens=none, parents=none, uniforms=none.float())
    with pytest.raises(ValueError, match="CUDA device"):  # as far as any valid call without a GPU
        mcpu.mcpu_verify_tree(**args)


@gpu
def test_a_batch_without_nodes():
    c = _case([0, 0, 0], 50, seed=26)
    got = _call(c)
    assert got[4] == 0 and not got[1].any() and np.all(got[2] == -1) and np.all(got[0] == -1) and not got[3].any()


def test_host_checks():
    from paper_2608_22167_gb300 import mcpu

    P, f = 1 << 20, mcpu._lib.mcpu_verify_tree
    ok = [P, 40, P, 40, 0, 40, P, P, P, P, P, P, 40, 3, 9, 4, P, P, P, P, P, None]
    assert f(*[0 if i == 13 else x for i, x in enumerate(ok)]) == 0  # no rows: nothing to do
    for i, bad in ((0, None), (0, P + 1), (1, 39), (3, 39), (4, 2), (5, 0), (6, None), (6, P + 2), (7, None), (8, None),
                   (9, P + 2), (10, None), (11, None), (12, 39), (13, -1), (14, -1), (15, 0), (16, None), (17, None),
                   (18, None), (19, P + 2), (20, None)):
        assert f(*[bad if k == i else x for k, x in enumerate(ok)]) == 1, (i, bad)
    assert f(*[2049 if k == 13 else x for k, x in enumerate(ok)]) == 2
    if not torch.cuda.is_available():
        assert f(*ok) == 4
