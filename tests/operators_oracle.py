"""Plain 64-bit numpy forms of the operators on token log probabilities and on gradients, and
the error bounds their kernels are held to."""
import numpy as np

U = 2.0 ** -24                                  # half a step of float32, relative
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 1e-37, "bfloat16": 1e-37, "float16": 2.0 ** -24}  # below the normal range


def rows(x, targets, live, scale, top):
    """x [N, V], targets [N] or None, live [N]: dict of what lfmmi_token_logprobs returns."""
    x = np.asarray(x, dtype=np.float64)
    N, V = x.shape
    out = {"logp": np.zeros(N), "entropy": np.zeros(N), "status": np.zeros(N, np.int32),
           "top_id": np.full((N, top), -1, np.int32), "top_logp": np.zeros((N, top)),
           "m": np.zeros(N), "logs": np.zeros(N), "l": np.full((N, V), -np.inf), "p": np.zeros((N, V))}
    for n in range(N):
        if not live[n]:
            continue
        bad = np.isnan(x[n]).any() or np.isposinf(x[n]).any()
        outside = targets is not None and targets[n] >= V
        out["status"][n] = 4 * outside
        if bad:
            out["status"][n] |= 2
            out["logp"][n] = out["entropy"][n] = out["m"][n] = out["logs"][n] = np.nan
            out["top_logp"][n] = np.nan
            continue
        order = np.lexsort((np.arange(V), -x[n]))[:top]
        out["top_id"][n] = order
        m = x[n].max()
        if m == -np.inf:
            out["status"][n] |= 1
            out["logp"][n] = np.nan if outside else -np.inf
            out["top_logp"][n] = out["m"][n] = out["logs"][n] = -np.inf
            continue
        with np.errstate(over="ignore"):
            d = scale * (x[n] - m)
            d = np.where(d < -np.finfo(np.float32).max, -np.inf, d)  # as float32 holds it
        s = np.exp(d).sum()
        l = d - np.log(s)
        p = np.exp(l)
        out["m"][n], out["logs"][n], out["l"][n], out["p"][n] = m, np.log(s), l, p
        out["entropy"][n] = -(p[p > 0] * l[p > 0]).sum()
        out["top_logp"][n] = l[order]
        if targets is not None:
            out["logp"][n] = np.nan if outside else l[targets[n]]
    return out


def grads(r, targets, live, scale, g, h):
    """Gradient [N, V] of sum(g * logp) + sum(h * entropy), from rows()'s answer `r`."""
    N, V = r["p"].shape
    out = np.zeros((N, V))
    for n in range(N):
        if not live[n] or r["status"][n]:
            continue
        p, l = r["p"][n], np.where(r["p"][n] > 0, r["l"][n], 0.0)
        out[n] = -scale * p * (g[n] + h[n] * (l + r["entropy"][n]))
        if targets is not None:
            out[n, targets[n]] += scale * g[n]
    return out


def loss(x, targets, scale, g, h):
    """sum(g * logp) + sum(h * entropy) of rows that are all live and finite somewhere."""
    r = rows(x, targets, np.ones(len(x), bool), scale, 0)
    return float((g * r["logp"]).sum() + (h * r["entropy"]).sum())


def bound_logs(V):
    """Of ln s. A difference to the maximum has 4 roundings (difference, two in the constant,
    product), so that a term exp(d) is off by 4 U |d| + 2 U, and the mean of |d| under p is at
    most ln V; where a lane's maximum moves its sum is multiplied by such a term, once for each of its
    V / 256 values at most, and as many additions round; the logarithm is off by 2 steps."""
    return U * (8.0 * np.log(V + 1.0) + 8.0 * (V // 256 + 1) + 24.0)


def bound_logp(V, l, d):
    return bound_logs(V) + 4.0 * U * np.abs(d) + 2.0 * U * np.abs(l)


def bound_entropy(V):
    """The mean of d under p: its terms carry the error of p and that of d, and the mean of d^2
    is at most (ln V)^2 + 2."""
    log = np.log(V + 1.0)
    return bound_logs(V) * (2.0 + log) + 8.0 * U * (log * log + 2.0)


def bound_grad(r, targets, scale, g, h, grad, dtype):
    """l is off by what ln s and d are, p by as much relatively; the sum and its products round
    8 times; the result is rounded to its type once. A p below the normal range, 2^-126, may be
    taken as 0: what is lost is at most 2^-126 times what p is multiplied by, g + h (|l| + H), where
    |l| is about 88 and more (2^-126 is e^-87.3)."""
    N, V = r["p"].shape
    p, l = r["p"], np.where(r["p"] > 0, r["l"], 0.0)
    d = l + np.where(np.isfinite(r["logs"]), r["logs"], 0.0)[:, None]
    off = bound_logp(V, l, d)
    g, h, ent = np.abs(g)[:, None], np.abs(h)[:, None], np.where(np.isfinite(r["entropy"]), r["entropy"], 0)[:, None]
    tol = p * (g + h * (np.abs(l) + ent)) * (off + 16 * U) + p * h * (off + bound_entropy(V))
    tol = tol + np.minimum(p, 2.0 ** -126) * (g + h * (np.abs(l) + ent))
    if targets is not None:
        at = np.clip(targets, 0, V - 1)
        tol[np.arange(N), at] += 4 * U * g[:, 0]
    return scale * tol + 1.001 * HALF[dtype] * np.abs(grad) + TINY[dtype]
