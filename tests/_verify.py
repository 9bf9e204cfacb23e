"""Plain verification of drafted trees (numpy, 64 bits), with the residual
carried as a vector: r <- max(r - m q, 0) after each rejection."""
import numpy as np


def softmax(x, heat):
    z = (x - x.max()) / heat
    e = np.exp(z)
    return e / e.sum()


def walk(logits, draft, tokens, parents, heat, u, noise, most):
    """One row: (path, next token, log-probabilities, how near the closest decision was to its border, relative)."""
    V = logits.shape[1]
    path, logp, margin = [0], [], np.inf
    while True:
        at = path[-1]
        x = logits[at].astype(np.float64)
        p = softmax(x, heat or 1.0)
        kids = [i for i in range(at + 1, len(tokens)) if parents[i] == at and 0 <= tokens[i] < V]
        kids = kids if len(path) < most else []
        went = None
        if heat == 0:
            pick = int(np.argmax(x))
            went = next((i for i in kids if tokens[i] == pick), None)
        else:
            r = p.copy()
            q = softmax(draft[at].astype(np.float64), heat) if draft is not None else None
            for i in kids:
                m = r.sum()
                level = r[tokens[i]] / (m * (q[tokens[i]] if q is not None else 1.0)) if m > 0 else 0.0
                margin = min(margin, abs(level - u[i]))
                if u[i] < level:
                    went = i
                    break
                if q is not None:
                    r = np.maximum(r - m * q, 0)
                else:
                    r[tokens[i]] = 0
            if went is None:
                race = (r if r.max() > 0 else p) / noise
                pick = int(np.argmax(race))
                rest = np.delete(race, pick)
                if rest.size:
                    margin = min(margin, 1 - rest.max() / race[pick])
        out = tokens[went] if went is not None else pick
        logp.append((x[out] - x.max()) / (heat or 1.0) - np.log(np.exp((x - x.max()) / (heat or 1.0)).sum()))
        if went is None:
            return path, pick, logp, margin
        path.append(went)


def reference(case):
    """Outputs of a whole batch, as mcpu_verify_tree lays them out."""
    rows, most = len(case["qsl"]) - 1, case["most"]
    path = np.full((rows, most), -1, np.int32)
    logp = np.zeros((rows, most))
    length, following, margin = np.zeros(rows, np.int32), np.full(rows, -1, np.int32), np.inf
    for r in range(rows):
        a, b = case["qsl"][r], case["qsl"][r + 1]
        if a == b:
            continue
        w, nxt, lp, near = walk(case["logits"][a:b], None if case["draft"] is None else case["draft"][a:b],
                                case["tokens"][a:b], case["parents"][a:b], case["heat"][r], case["u"][a:b],
                                case["noise"][r], most)
        path[r, : len(w)], logp[r, : len(w)] = w, lp
        length[r], following[r], margin = len(w), nxt, min(margin, near)
    return path, length, following, logp, margin
