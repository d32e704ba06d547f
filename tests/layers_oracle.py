"""Plain 64-bit numpy forms of the operators around an output layer (embeddings, dropout, the end
of a residual block, verification of drafted tokens), and the error bounds their kernels are held to."""
import numpy as np

U = 2.0 ** -24                                  # half a step of float32, relative
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 1e-37, "bfloat16": 1e-37, "float16": 2.0 ** -24}  # below the normal range


def rounding(dtype):
    """Of a value that is rounded to `dtype` once (from fp32: for float32 that has happened)."""
    return 0.0 if dtype == "float32" else 1.001 * HALF[dtype]


# ---- embeddings

def embed(table, tokens, live, scale):
    """table [V, D], tokens [N], live [N]: (rows [N, D], status [N])."""
    V = table.shape[0]
    out = np.zeros((len(tokens), table.shape[1]))
    status = np.zeros(len(tokens), np.int32)
    for n, t in enumerate(tokens):
        if not live[n] or t < 0:
            continue
        status[n] = 4 * (t >= V)
        out[n] = np.nan if t >= V else scale * table[t]
    return out, status


def embed_grad(g, tokens, live, scale, V):
    """(gradient [V, D], sums of |g| [V, D], positions of each token [V])."""
    grad, size, count = np.zeros((V, g.shape[1])), np.zeros((V, g.shape[1])), np.zeros(V, np.int64)
    ok = live & (tokens >= 0) & (tokens < V)
    np.add.at(grad, tokens[ok], g[ok])
    np.add.at(size, tokens[ok], np.abs(g[ok]))
    np.add.at(count, tokens[ok], 1)
    return scale * grad, scale * size, count


def bound_embed_grad(want, size, count, dtype, old=None):
    """Of c values added in any order every one goes through at most c - 1 additions; one more
    rounding each for the scale, an addition to `old`, and the type."""
    tol = size * U * (count[:, None] + 1.0) + U * np.abs(want) + rounding(dtype) * np.abs(want) + TINY[dtype]
    return tol if old is None else tol + U * np.abs(old) * 2


# ---- dropout

def philox(counter, key):
    """Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3,
    SC 2011) in whole numbers without a size."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def threshold(p):
    return int(np.rint(float(np.float32(p)) * 65536.0))


def words(chunks, rows, draw, seed):
    """philox of the counters (chunk, row, draw), arrays of whole numbers: [..., 4]."""
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    chunks, rows = np.broadcast_arrays(np.asarray(chunks, np.uint64), np.asarray(rows, np.uint64))
    draw &= (1 << 64) - 1
    c = [chunks, rows, np.full_like(chunks, draw & 0xFFFFFFFF), np.full_like(chunks, draw >> 32)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, -1)


def kept(rows, D, p, seed, draw):
    """[len(rows), D] truth values; rows: row numbers."""
    w = words(np.arange((D + 7) // 8)[None], np.asarray(rows)[:, None], draw, seed)
    halves = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1)
    return halves.reshape(len(rows), -1)[:, :D] >= threshold(p)


def factor(p):
    k = threshold(p)
    return 0.0 if k == 65536 else 65536.0 / (65536 - k)


def dropped(x, mask, p):
    return np.where(mask, x, 0.0) * factor(p)


def bound_dropped(want, dtype):
    """The factor and the product are rounded, then the type."""
    return np.abs(want) * (2.1 * U + rounding(dtype)) + TINY[dtype]


# ---- the end of a residual block

def adds(D):
    """Most additions that a value goes through in a sum over a row: a lane's own, 64 lanes', 16
    waves' at most."""
    return 32 + (D + 8191) // 8192 * 8 + 8 + 16


def norm(total, weight, eps):
    """total [N, D] as it is kept: (y, rstd [N])."""
    rstd = 1.0 / np.sqrt((total * total).mean(1) + eps)
    return total * rstd[:, None] * weight, rstd


def bound_rstd(D):
    """Relative: squares and sum err by `adds` + 1 steps, the mean and eps by 2 more, the root
    halves that; root and quotient round."""
    return U * ((adds(D) + 3) / 2.0 + 2.0)


def bound_norm(y, D, dtype):
    return np.abs(y) * (bound_rstd(D) + 2.1 * U + rounding(dtype)) + TINY[dtype]


def bytes_scale(y):
    return np.maximum(np.abs(y).max(1) / 448.0, 2.0 ** -126)


def bound_bytes(v, off):
    """v / scale rounded to e4m3 (three bits behind the leading one, from 2^-6 down steps of 2^-9),
    `off`: how far the quotient is off before, relatively."""
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -9)))
    step = 2.0 ** (np.maximum(e, -6.0) - 3.0)
    return step / 2.0 + off * np.abs(v) + 1e-30


def norm_grads(total, rstd, weight, dy, dsum):
    """(d [N, D], gradient of the weight [D]) for rstd as the kernel is given it."""
    n = total * rstd[:, None]
    g = dy * weight
    d = dsum + rstd[:, None] * (g - n * (g * n).mean(1, keepdims=True))
    return d, (dy * n).sum(0)


def bound_norm_grads(total, rstd, weight, dy, dsum, d, dw, dtype, weight_dtype):
    """n and g are rounded once; the mean of g n errs by `adds` + 4 steps of the mean of |g n|; two
    products and the difference, times rstd, added. dw: a value goes through at most all its
    rows' additions and 64 more of partial sums."""
    D, rows = total.shape[1], total.shape[0]
    n, g = np.abs(total * rstd[:, None]), np.abs(dy * weight)
    mean = (g * n).mean(1, keepdims=True)
    tol = rstd[:, None] * (2 * U * g + n * mean * U * (adds(D) + 9)) + U * (2 * np.abs(d) + np.abs(dsum))
    tol_w = (np.abs(dy) * n).sum(0) * U * (rows + 66)
    return tol + rounding(dtype) * (np.abs(d) + tol) + TINY[dtype], \
        tol_w + rounding(weight_dtype) * (np.abs(dw) + tol_w) + TINY[weight_dtype]


def norm_loss(x, residual, weight, eps, mask, p, wy, ws):
    """sum(wy * y) + sum(ws * sum) with nothing rounded."""
    total = residual + dropped(x, mask, p)
    return float((wy * norm(total, weight, eps)[0]).sum() + (ws * total).sum())


# ---- drafted tokens

def softmax(x, scale):
    """(probabilities, flag) of a row."""
    if np.isnan(x).any() or np.isposinf(x).any():
        return None, 2
    if np.isneginf(x).all():
        return None, 1
    with np.errstate(over="ignore"):
        d = (x - x.max()) * float(np.float32(scale))
    e = np.where(d > -1000.0 * np.log(2.0), np.exp(np.maximum(d, -700.0)), 0.0)
    return e / e.sum(), 0


def draw(weights, u):
    """The first index at which the running sum passes u times the whole."""
    cum = np.cumsum(weights)
    over = np.flatnonzero((cum > float(u) * cum[-1]) & (weights > 0))
    return int(over[0]) if len(over) else int(np.flatnonzero(weights > 0)[-1])


def verify(logits, drafted, n, scale, uniforms=None, draft=None, draft_scale=1.0):
    """One sequence: logits [K + 1, V], drafted [K], uniforms [K + 1] or None, draft [K, V] or None.
    (accepted, token or -1, status)."""
    V = logits.shape[1]
    for i in range(n + 1):
        p, flag = softmax(logits[i], scale)
        if i < n:
            d = int(drafted[i])
            q = None
            if draft is not None and uniforms is not None:
                q, other = softmax(draft[i], draft_scale)
                flag |= other
            if not 0 <= d < V:
                flag |= 4
        if flag:
            return i, -1, flag
        if uniforms is None:
            best = int(np.argmax(logits[i]))
            if i < n and d == best:
                continue
            return i, best, 0
        if i < n:
            if q is None:
                q = np.zeros(V)
                q[d] = 1.0
            if float(uniforms[i]) * q[d] < p[d]:
                continue
            rest = np.maximum(p - q, 0.0)
            return i, draw(rest if rest.sum() > 0 else p, uniforms[-1]), 0
        return n, draw(p, uniforms[-1]), 0
