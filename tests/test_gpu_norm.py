"""Dropout, and the end of a residual block (the residual's addition with a root-mean-square norm),
against the 64-bit forms."""
import numpy as np
import pytest

from paper_2005_09824_amd import binding, chain
from tests import layers_oracle as oracle

pytestmark = pytest.mark.gpu

DTYPES = ["float32", "bfloat16", "float16"]
WIDTHS = [1, 2, 7, 8, 9, 63, 64, 65, 84, 511, 512, 513, 640, 1000, 1024, 1025, 2047, 2048, 2049, 4096, 4099, 5003, 8192, 8193,
          16384, 16391, 32771]


def _torch():
    import torch
    return torch


def _name(t):
    return str(t.dtype).replace("torch.", "")


def _values(rng, shape, dtype, sigma=1.0):
    """(device tensor, its values in 64 bits)"""
    torch = _torch()
    x = torch.from_numpy(rng.normal(0, sigma, shape).astype(np.float32)).to(getattr(torch, dtype)).cuda()
    return x, x.double().cpu().numpy()


def _host(t):
    return t.double().cpu().numpy()


def _close(got, want, tol, what):
    got = _host(got).reshape(want.shape)
    off, tol = np.abs(got - want), np.broadcast_to(tol, want.shape)
    assert np.all(off <= tol), (what, off.max(), (off / np.maximum(tol, 1e-300)).max())


# ---- dropout

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [1, 3, 8, 9, 64, 65, 255, 2047, 2048, 2049, 8193, 100003])
def test_dropout(D, dtype):
    rng = np.random.default_rng(D)
    R = 37 if D < 3000 else 3
    x, x64 = _values(rng, (R, D), dtype)
    for p, seed, offset in ((0.1, 1, 0), (0.5, (1 << 63) + 5, (1 << 64) - 1), (0.0, 3, 4), (1.0, 3, 4)):
        y = binding.lfmmi_dropout(x, p, seed, offset)
        mask = oracle.kept(np.arange(R), D, p, seed, offset)
        want = oracle.dropped(x64, mask, p)
        _close(y, want, oracle.bound_dropped(want, dtype), "dropout")
        assert not _host(y)[~mask].any()


def test_shares_of_what_is_dropped():
    # 4 million independent choices: within 6 deviations of p, in all, by column in a block, and of neighbours
    torch = _torch()
    x = torch.ones((2048, 2048), device="cuda")
    for p in (0.05, 0.3):
        zero = (binding.lfmmi_dropout(x, p, 77, 5) == 0).double()
        assert abs(float(zero.mean()) - p) < 6 * (p * (1 - p) / zero.numel()) ** 0.5 + 2.0 ** -17
        per = zero.reshape(2048, 256, 8).mean((0, 1))
        assert float((per - p).abs().max()) < 6 * (p * (1 - p) * 8 / zero.numel()) ** 0.5 + 2.0 ** -17
        for other in (zero.roll(1, 0), zero.roll(1, 1), zero.roll(8, 1), (binding.lfmmi_dropout(x, p, 77, 6) == 0).double(),
                      (binding.lfmmi_dropout(x, p, 78, 5) == 0).double()):
            both = float((zero * other).mean())
            assert abs(both - p * p) < 6 * (p * p / zero.numel()) ** 0.5 + 2.0 ** -16


@pytest.mark.parametrize("dtype", DTYPES)
def test_dropout_layouts(dtype):
    torch = _torch()
    rng = np.random.default_rng(4)
    x, x64 = _values(rng, (3, 5, 4, 33), dtype)
    mask = oracle.kept(np.arange(60), 33, 0.25, 9, 2).reshape(3, 5, 4, 33)
    want = oracle.dropped(x64, mask, 0.25)
    tol = oracle.bound_dropped(want, dtype)
    _close(binding.lfmmi_dropout(x, 0.25, 9, 2), want, tol, "four dimensions")
    base = torch.full((60, 40), float("nan"), dtype=x.dtype, device="cuda")
    view = base[:, 3:36]
    view.copy_(x.reshape(60, 33))
    _close(binding.lfmmi_dropout(view, 0.25, 9, 2), want.reshape(60, 33), tol.reshape(60, 33), "a view")
    assert torch.isnan(base[:, :3]).all() and torch.isnan(base[:, 36:]).all()
    version = base._version
    assert binding.lfmmi_dropout(view, 0.25, 9, 2, out=view) is view   # in place: what lies around it stays
    _close(view, want.reshape(60, 33), tol.reshape(60, 33), "in place")
    assert torch.isnan(base[:, :3]).all() and torch.isnan(base[:, 36:]).all() and base._version > version
    out = torch.empty_like(x)
    assert binding.lfmmi_dropout(x, 0.25, 9, 2, out=out) is out
    _close(out, want, tol, "out")
    one = x[0, 0, 0]
    _close(binding.lfmmi_dropout(one, 0.25, 9, 2), want[0, 0, 0], tol[0, 0, 0], "one row")
    same = one.expand(60, 33)
    _close(binding.lfmmi_dropout(same, 0.25, 9, 2), oracle.dropped(np.broadcast_to(x64[0, 0, 0], (60, 33)), mask.reshape(60, 33), 0.25),
           oracle.bound_dropped(np.broadcast_to(x64[0, 0, 0], (60, 33)) * 2, dtype), "one row for all")
    assert binding.lfmmi_dropout(x[:0], 0.25, 9).shape == (0, 5, 4, 33) and binding.lfmmi_dropout(x[..., :0], 0.25, 9).numel() == 0
    with pytest.raises(ValueError):
        binding.lfmmi_dropout(x.transpose(0, 1), 0.25, 9)
    with pytest.raises(ValueError):
        binding.lfmmi_dropout(x, 0.25, 9, out=out[:2])
    with pytest.raises(binding.LfmmiError):
        binding.lfmmi_dropout(same, 0.25, 9, out=same)
    for kw in (dict(p=1.5), dict(p=-0.1), dict(seed=-1), dict(seed=1 << 64), dict(offset=-1), dict(step=torch.zeros(1, device="cuda")),
               dict(step=torch.zeros(2, dtype=torch.int64, device="cuda"))):
        with pytest.raises(ValueError):
            binding.lfmmi_dropout(x, **dict(dict(p=0.1, seed=1), **kw))


def test_dropped_values_are_zero_whatever_they_were():
    torch = _torch()
    x = torch.full((50, 50), float("nan"), device="cuda")
    x[::2] = float("inf")
    y = binding.lfmmi_dropout(x, 0.5, 3)
    mask = oracle.kept(np.arange(50), 50, 0.5, 3, 0)
    assert not _host(y)[~mask].any() and not np.isfinite(_host(y)[mask]).any()
    assert not binding.lfmmi_dropout(x, 1.0, 3).any()


def test_a_step_on_the_device_moves_the_draw():
    torch = _torch()
    x = torch.ones((20, 100), device="cuda")
    step = torch.tensor([7], device="cuda")
    assert torch.equal(binding.lfmmi_dropout(x, 0.3, 5, 2, step), binding.lfmmi_dropout(x, 0.3, 5, 9))
    step.fill_(-3)   # modulo 2^64
    assert torch.equal(binding.lfmmi_dropout(x, 0.3, 5, 2, step), binding.lfmmi_dropout(x, 0.3, 5, (1 << 64) - 1))
    graph, y = torch.cuda.CUDAGraph(), torch.empty_like(x)
    step.fill_(0)
    with torch.cuda.graph(graph):
        binding.lfmmi_dropout(x, 0.3, 5, 2, step, out=y)
        step.add_(1)
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, binding.lfmmi_dropout(x, 0.3, 5, 2 + k))


@pytest.mark.parametrize("dtype", DTYPES)
def test_dropout_through_autograd(dtype):
    torch = _torch()
    rng = np.random.default_rng(6)
    x, x64 = _values(rng, (6, 5, 21), dtype)
    x.requires_grad_()
    g, g64 = _values(rng, (6, 5, 21), dtype)
    mask = oracle.kept(np.arange(30), 21, 0.4, 1, 2).reshape(6, 5, 21)
    y = chain.dropout(x, 0.4, 1, 2)
    (grad,) = torch.autograd.grad(y, x, g)
    for got, v in ((y.detach(), x64), (grad, g64)):
        want = oracle.dropped(v, mask, 0.4)
        _close(got, want, oracle.bound_dropped(want, dtype), "dropout")
    # rows in another order of memory are rows all the same
    y = chain.dropout(x.transpose(0, 1), 0.4, 1, 2)
    want = oracle.dropped(x64.transpose(1, 0, 2), oracle.kept(np.arange(30), 21, 0.4, 1, 2).reshape(5, 6, 21), 0.4)
    _close(y.detach(), want, oracle.bound_dropped(want, dtype), "transposed")
    (grad,) = torch.autograd.grad(y.sum(), x)
    assert np.array_equal(_host(grad) != 0, oracle.kept(np.arange(30), 21, 0.4, 1, 2).reshape(5, 6, 21).transpose(1, 0, 2))
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    y = chain.dropout(x, 0.4, 1, 2, step)
    step.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


# ---- the end of a residual block

def check_norm(x64, r64, weight, eps, lengths, p, seed, draw, r, dtype, shape):
    """`r`: the call's answer for rows x64 (+ r64) of `shape`."""
    D = shape[-1]
    N = int(np.prod(shape[:-1]))
    B, T = (shape[0], shape[1]) if len(shape) == 3 else (shape[0], 1)
    live = np.ones((B, T), bool)
    if lengths is not None:
        live &= np.arange(T)[None] < np.asarray(lengths)[:, None]
    live = live.reshape(-1)[:, None]
    h = x64.reshape(N, D)
    tol = np.zeros_like(h)
    if p > 0:
        h = oracle.dropped(h, oracle.kept(np.arange(N), D, p, seed, draw), p)
        tol = np.abs(h) * 2.1 * oracle.U
    if r64 is not None:
        h = h + r64.reshape(N, D)
        tol = tol + np.abs(h) * oracle.U
    if p > 0 or r64 is not None:
        tol = tol + np.abs(h) * oracle.rounding(dtype) + oracle.TINY[dtype]
        _close(r.sum, np.where(live, h, 0.0), tol * live, "sum")
    total = _host(r.sum).reshape(N, D) * live
    w = np.ones(D) if weight is None else _host(weight)
    y, rstd = oracle.norm(total, w, float(np.float32(eps)))
    y, rstd = y * live, rstd * live[:, 0]
    _close(r.rstd, rstd, rstd * oracle.bound_rstd(D), "rstd")
    if r.y is not None:
        _close(r.y, y, oracle.bound_norm(y, D, dtype) * live, "y")
    if r.q is not None:
        scale = oracle.bytes_scale(y) * live[:, 0]
        off = 2 * oracle.bound_rstd(D) + 10 * oracle.U
        _close(r.q_scale, scale, scale * off, "q_scale")
        v = y / np.where(live, scale[:, None], 1.0)
        _close(r.q.float(), v, oracle.bound_bytes(v, off) * live, "q")
    return total, w


def check_grads(total, w, rstd, dy, dsum, lengths, p, seed, draw, g, dtype, weight_dtype, shape):
    D = shape[-1]
    N = int(np.prod(shape[:-1]))
    B, T = (shape[0], shape[1]) if len(shape) == 3 else (shape[0], 1)
    live = np.ones((B, T), bool)
    if lengths is not None:
        live &= np.arange(T)[None] < np.asarray(lengths)[:, None]
    live = live.reshape(-1)[:, None]
    zero = np.zeros((N, D))
    dy = zero if dy is None else np.where(live, dy.reshape(N, D), 0.0)
    dsum = zero if dsum is None else np.where(live, dsum.reshape(N, D), 0.0)
    rstd = _host(rstd).reshape(N)
    d, dw = oracle.norm_grads(total, rstd, w, dy, dsum)
    tol, tol_w = oracle.bound_norm_grads(total, rstd, w, dy, dsum, d, dw, dtype, weight_dtype or "float32")
    if g.residual is not None:
        _close(g.residual, d, tol * live, "gradient of the residual")
    want, tol_x = d, tol
    if p > 0:
        mask = oracle.kept(np.arange(N), D, p, seed, draw)
        want = oracle.dropped(d, mask, p)
        tol_x = np.where(mask, tol * oracle.factor(p), 0.0) + np.abs(want) * 2.1 * oracle.U
    _close(g.x, want, tol_x * live, "gradient of x")
    if g.weight is not None:
        _close(g.weight, dw, tol_w, "gradient of the weight")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", WIDTHS)
def test_norm(D, dtype):
    torch = _torch()
    rng = np.random.default_rng(D)
    N = 23 if D < 3000 else 5
    x, x64 = _values(rng, (N, D), dtype)
    res, r64 = _values(rng, (N, D), dtype, 3.0)
    dy, dy64 = _values(rng, (N, D), dtype)
    ds, ds64 = _values(rng, (N, D), dtype)
    for p, residual, w_dtype, quantized in ((0.0, True, "float32", False), (0.2, True, dtype, True), (0.0, False, "float32", True),
                                            (0.2, False, None, False)):
        weight = None
        if w_dtype:
            weight = torch.from_numpy(rng.normal(1, 0.3, D).astype(np.float32)).to(getattr(torch, w_dtype)).cuda()
        kw = dict(p=p, seed=11, offset=D)
        r = binding.lfmmi_add_rms_norm(x, res if residual else None, weight, eps=1e-5, quantized=quantized,
                                       y="both" if quantized else True, **kw)
        total, w = check_norm(x64, r64 if residual else None, weight, 1e-5, None, p, 11, D, r, dtype, (N, D))
        g = binding.lfmmi_add_rms_norm_backward(r.sum, r.rstd, weight, dy, ds if residual else None, residual=residual, **kw)
        check_grads(total, w, r.rstd, dy64, ds64 if residual else None, None, p, 11, D, g, dtype, w_dtype, (N, D))
        only = binding.lfmmi_add_rms_norm_backward(r.sum, r.rstd, weight, None, ds, residual=residual, **kw)
        check_grads(total, w, r.rstd, None, ds64, None, p, 11, D, only, dtype, w_dtype, (N, D))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [513, 1024, 1100, 2048, 2100, 3001, 4096, 5003, 8192])
def test_norm_of_many_rows(D, dtype):
    # (few rows are spread over more lanes each)
    torch = _torch()
    rng = np.random.default_rng(D)
    N = 523
    x, x64 = _values(rng, (N, D), dtype)
    res, r64 = _values(rng, (N, D), dtype, 3.0)
    weight = torch.from_numpy(rng.normal(1, 0.3, D).astype(np.float32)).cuda()
    for p, quantized in ((0.0, True), (0.2, False)):
        r = binding.lfmmi_add_rms_norm(x, res, weight, p=p, seed=3, offset=4, quantized=quantized, y="both" if quantized else True)
        check_norm(x64, r64, weight, 1e-6, None, p, 3, 4, r, dtype, (N, D))
    few = binding.lfmmi_add_rms_norm(x[:300], res[:300], weight, p=0.2, seed=3, offset=4)
    assert torch.equal(few.sum, r.sum[:300])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,D", [(1100, 1201), (520, 1536), (1100, 2001), (1600, 2501), (1600, 3064), (520, 5113), (520, 6000), (1040, 6001),
                                 (520, 6145), (520, 7001), (520, 9001), (520, 12288), (520, 12289), (520, 16000)])
def test_norm_and_gradients_of_more_rows_than_workgroups(N, D, dtype):
    torch = _torch()
    rng = np.random.default_rng(D)
    x, x64 = _values(rng, (N, D), dtype)
    res, r64 = _values(rng, (N, D), dtype, 3.0)
    dy, dy64 = _values(rng, (N, D), dtype)
    weight = torch.from_numpy(rng.normal(1, 0.3, D).astype(np.float32)).cuda()
    kw = dict(p=0.2, seed=3, offset=4)
    r = binding.lfmmi_add_rms_norm(x, res, weight, **kw)
    total, w = check_norm(x64, r64, weight, 1e-6, None, 0.2, 3, 4, r, dtype, (N, D))
    g = binding.lfmmi_add_rms_norm_backward(r.sum, r.rstd, weight, dy, x, **kw)
    check_grads(total, w, r.rstd, dy64, x64, None, 0.2, 3, 4, g, dtype, "float32", (N, D))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,T,D", [(1, 1, 16), (5, 7, 40), (300, 3, 24), (600, 1, 640), (4, 700, 72), (3, 40, 2100), (2, 9, 16400),
                                   (1, 3000, 16), (280, 2, 20000)])
def test_sequences(B, T, D, dtype):
    # lengths of zero, of one and of all; what lies behind them is NaN
    torch = _torch()
    rng = np.random.default_rng(B + T + D)
    lengths = rng.integers(0, T + 1, B)
    lengths[: min(B, 3)] = [0, 1, T][: min(B, 3)] if B >= 3 else [T] * min(B, 3)
    x, x64 = _values(rng, (B, T, D), dtype)
    res, r64 = _values(rng, (B, T, D), dtype)
    dy, dy64 = _values(rng, (B, T, D), dtype)
    ds, ds64 = _values(rng, (B, T, D), dtype)
    behind = np.arange(T)[None] >= lengths[:, None]
    for t in (x, res, dy, ds):
        t[torch.from_numpy(behind).cuda()] = float("nan")
    for v in (x64, r64):
        v[behind] = 0.0
    weight = torch.from_numpy(rng.normal(1, 0.3, D).astype(np.float32)).cuda()
    kw = dict(lengths=lengths, p=0.3, seed=5, offset=6)
    r = binding.lfmmi_add_rms_norm(x, res, weight, quantized=True, y="both", **kw)
    total, w = check_norm(x64, r64, weight, 1e-6, lengths, 0.3, 5, 6, r, dtype, (B, T, D))
    g = binding.lfmmi_add_rms_norm_backward(r.sum, r.rstd, weight, dy, ds, **kw)
    check_grads(total, w, r.rstd, dy64, ds64, lengths, 0.3, 5, 6, g, dtype, "float32", (B, T, D))
    again = binding.lfmmi_add_rms_norm_backward(r.sum, r.rstd, weight, dy, ds, **kw)
    assert all(torch.equal(a, b) for a, b in zip(g, again))
    # a norm of x itself reads nothing behind its lengths either
    r = binding.lfmmi_add_rms_norm(x, None, weight, lengths=lengths)
    assert r.sum is x
    total, w = check_norm(x64, None, weight, 1e-6, lengths, 0.0, 0, 0, r._replace(sum=torch.from_numpy(x64)), dtype, (B, T, D))
    g = binding.lfmmi_add_rms_norm_backward(x, r.rstd, weight, dy, lengths=lengths, residual=False)
    check_grads(total, w, r.rstd, dy64, None, lengths, 0.0, 0, 0, g, dtype, "float32", (B, T, D))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [33, 700, 5001, 20001])
def test_views_and_places(D, dtype):
    torch = _torch()
    rng = np.random.default_rng(D)
    B, T = 2, 3
    base = torch.full((B, T + 2, D + 9), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    x = base[:, 1:T + 1, 5:5 + D]
    x.copy_(torch.from_numpy(rng.normal(0, 1, (B, T, D)).astype(np.float32)))
    res, r64 = _values(rng, (1, 1, D), dtype)
    weight = torch.from_numpy(rng.normal(1, 0.3, D).astype(np.float32)).cuda()
    r = binding.lfmmi_add_rms_norm(x, res.expand(B, T, D), weight)   # a residual that is one row for all
    check_norm(_host(x), np.broadcast_to(r64, (B, T, D)), weight, 1e-6, None, 0.0, 0, 0, r, dtype, (B, T, D))
    alone = binding.lfmmi_add_rms_norm(x, None, weight)
    assert alone.sum is x
    total, w = check_norm(_host(x), None, weight, 1e-6, None, 0.0, 0, 0, alone, dtype, (B, T, D))
    dy, dy64 = _values(rng, (B, T, D), dtype)
    g = binding.lfmmi_add_rms_norm_backward(x, alone.rstd, weight, dy, residual=False)
    check_grads(total, w, alone.rstd, dy64, None, None, 0.0, 0, 0, g, dtype, "float32", (B, T, D))
    # sums in the place of an input, gradients in the place of those that come in: the same bits
    kw = dict(p=0.2, seed=1, offset=2)
    res, r64 = _values(rng, (B, T, D), dtype)
    xc = x.contiguous()
    want = binding.lfmmi_add_rms_norm(xc, res, weight, quantized=True, **kw)
    for place in ("x", "residual"):
        a, b = xc.clone(), res.clone()
        out = binding.AddRmsNorm(a if place == "x" else b, None, *(torch.empty_like(t) for t in want[2:]))
        got = binding.lfmmi_add_rms_norm(a, b, weight, quantized=True, out=out, **kw)
        assert got.sum is out.sum and torch.equal(got.sum, want.sum) and torch.equal(got.rstd, want.rstd)
        assert torch.equal(got.q.view(torch.uint8), want.q.view(torch.uint8)) and torch.equal(got.q_scale, want.q_scale)
    twice = binding.lfmmi_add_rms_norm(xc, xc, weight)
    a = xc.clone()
    got = binding.lfmmi_add_rms_norm(a, a, weight, out=binding.AddRmsNorm(a, *(torch.empty_like(t) for t in twice[1:3]), None, None))
    assert torch.equal(got.sum, twice.sum) and torch.equal(got.y, twice.y)
    ds, ds64 = _values(rng, (B, T, D), dtype)
    want_g = binding.lfmmi_add_rms_norm_backward(want.sum, want.rstd, weight, dy, ds, **kw)
    for swap in (False, True):
        a, b = dy.clone(), ds.clone()
        dw = torch.empty_like(weight)
        out = binding.AddRmsNormGrads(*((b, a) if swap else (a, b)), dw)
        got = binding.lfmmi_add_rms_norm_backward(want.sum, want.rstd, weight, a, b, out=out, **kw)
        assert got.x is out.x and all(torch.equal(s, t) for s, t in zip(got, want_g))
    with pytest.raises(binding.LfmmiError):
        binding.lfmmi_add_rms_norm(xc, res, weight, out=binding.AddRmsNorm(want.sum, want.sum, want.rstd, None, None))
    with pytest.raises(ValueError):
        binding.lfmmi_add_rms_norm(xc, res, weight, out=binding.AddRmsNorm(None, torch.empty_like(xc), want.rstd, None, None))
    with pytest.raises(ValueError):
        binding.lfmmi_add_rms_norm(xc, res[:, :2], weight)
    with pytest.raises(ValueError):
        binding.lfmmi_add_rms_norm(xc, res, weight[:-1])


def test_one_tensor_for_both_gradients():
    # without dropout they are the same; with it, one tensor cannot hold both
    torch = _torch()
    x, dy = torch.randn((4, 30), device="cuda"), torch.randn((4, 30), device="cuda")
    r = binding.lfmmi_add_rms_norm(x, x)
    pair = binding.lfmmi_add_rms_norm_backward(r.sum, r.rstd, None, dy)
    assert pair.x is pair.residual
    assert binding.lfmmi_add_rms_norm_backward(r.sum, r.rstd, None, dy, out=pair) is pair
    dropped = dict(p=0.5, seed=1)
    r = binding.lfmmi_add_rms_norm(x, x, **dropped)
    before = pair.x.clone()
    with pytest.raises(ValueError, match="one tensor"):
        binding.lfmmi_add_rms_norm_backward(r.sum, r.rstd, None, dy, out=pair, **dropped)
    with pytest.raises(binding.LfmmiError):
        binding.lfmmi_add_rms_norm_backward(r.sum, r.rstd, None, dy, out=pair._replace(residual=pair.x.view(4, 30)), **dropped)
    assert torch.equal(pair.x, before)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [40, 3000, 20000])
def test_rows_of_zeros_and_values_that_are_none(D, dtype):
    torch = _torch()
    x = torch.randn((6, D), dtype=torch.float32, device="cuda").to(getattr(torch, dtype))
    x[1] = 0.0
    x[2, D // 2] = float("nan")
    x[3, D - 1] = float("inf")
    x[4] = torch.finfo(x.dtype).max if dtype == "float16" else 1e18
    r = binding.lfmmi_add_rms_norm(x, None, quantized=True, y="both")
    y, q, scale = r.y.float(), r.q.float(), r.q_scale
    assert not y[1].any() and not q[1].any() and float(scale[1]) == 2.0 ** -126
    assert torch.isnan(y[2]).all() and torch.isnan(q[2]).all() and torch.isnan(scale[2])
    assert torch.isnan(y[3, D - 1]) and not y[3, : D - 1].any() and torch.isnan(scale[3])
    assert torch.allclose(y[4], torch.ones_like(y[4]), rtol=1e-2) and float(q[4].min()) == 448.0
    for i in (0, 5):
        assert torch.isfinite(y[i]).all() and float(q[i].abs().max()) == 448.0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [128, 700, 5003, 20000])
def test_bytes_next_to_a_tie(D, dtype):
    # rows of 1: y is the weight, to the bit. Weights that are halfway between two e4m3 values times a scale of 17
    # bits: the quotient is that halfway value, which goes to the even one of the two
    torch = _torch()
    ties = np.array([m * 2.0 ** e for m in range(17, 32, 2) for e in range(-6, 4)] + [448.0])
    want = torch.from_numpy(np.tile(ties, D // len(ties) + 1)[:D] * np.where(np.arange(D) % 3 == 0, -1.0, 1.0))
    want[0] = 448.0
    x = torch.ones((1, D), dtype=getattr(torch, dtype), device="cuda")
    rng = np.random.default_rng(D)
    for exponent in (-142, -141, -100, -77, -76, -75, 100, *range(-30, -10)):   # (2^-126 is the least scale)
        scale = float(rng.integers(1 << 16, 1 << 17)) * 2.0 ** exponent
        weight = (want * scale).float().cuda()
        assert torch.equal(weight.double().cpu(), want * scale)
        r = binding.lfmmi_add_rms_norm(x, None, weight, eps=1e-30, quantized=True)
        assert float(r.rstd) == 1.0 and float(r.q_scale) == scale
        assert torch.equal(r.q[0].float().cpu(), want.float().to(torch.float8_e4m3fn).float())


@pytest.mark.parametrize("D", [40, 3000, 20000])
def test_bytes_of_values_beyond_the_type(D):
    # a weight that takes a value to infinity: the scale is that, what is finite over it 0, infinity over it NaN
    torch = _torch()
    x = torch.ones((2, D), device="cuda")
    weight = torch.full((D,), -3.0, device="cuda")
    weight[D // 3] = 3e38
    x[0, D // 3] = 4.0
    r = binding.lfmmi_add_rms_norm(x, None, weight, quantized=True, y="both")
    q = r.q.float()
    assert torch.isinf(r.y[0, D // 3]) and torch.isinf(r.q_scale[0]) and torch.isnan(q[0, D // 3])
    q[0, D // 3] = 0
    assert not q[0].any() and float(q[1, D // 3]) == 448.0


def test_eps_beside_squares_that_overflow():
    # 2^20 squares of 4e32 are beyond fp32 together; the largest eps is nothing beside their mean
    torch = _torch()
    rng = np.random.default_rng(12)
    x, x64 = _values(rng, (2, 1 << 20), "float32", 2e16)
    r = binding.lfmmi_add_rms_norm(x, None, None, eps=1e20)
    check_norm(x64, None, None, 1e20, None, 0.0, 0, 0, r, "float32", x.shape)


def test_norm_of_no_rows():
    torch = _torch()
    weight = torch.ones(8, device="cuda")
    for shape in ((0, 8), (0, 3, 8), (3, 0, 8)):
        x = torch.zeros(shape, device="cuda")
        r = binding.lfmmi_add_rms_norm(x, x, weight, p=0.5)
        assert r.y.shape == shape
        g = binding.lfmmi_add_rms_norm_backward(r.sum, r.rstd, weight, x, x, p=0.5)
        assert g.x.shape == shape and not g.weight.any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_norm_through_autograd(p, dtype):
    torch = _torch()
    rng = np.random.default_rng(21)
    B, T, D = 3, 6, 50
    lengths = [6, 0, 4]
    x, x64 = _values(rng, (B, T, D), dtype)
    res, r64 = _values(rng, (B, T, D), dtype)
    weight = torch.from_numpy(rng.normal(1, 0.3, D).astype(np.float32)).cuda()
    for t in (x, res, weight):
        t.requires_grad_()
    y, total = chain.add_rms_norm(x, res, weight, 1e-5, lengths, p, 3, 4)
    r = binding.lfmmi_add_rms_norm(x.detach(), res.detach(), weight.detach(), 1e-5, lengths, p, 3, 4)
    assert torch.equal(y, r.y) and torch.equal(total, r.sum)
    dy, dy64 = _values(rng, (B, T, D), dtype)
    ds, ds64 = _values(rng, (B, T, D), dtype)
    got = torch.autograd.grad((y, total), (x, res, weight), (dy, ds), retain_graph=True)
    check_grads(_host(r.sum).reshape(-1, D), _host(weight.detach()), r.rstd, dy64, ds64, lengths, p, 3, 4,
                binding.AddRmsNormGrads(*got), dtype, "float32", (B, T, D))
    got = torch.autograd.grad(y, (x, res, weight), dy, retain_graph=True)
    check_grads(_host(r.sum).reshape(-1, D), _host(weight.detach()), r.rstd, dy64, None, lengths, p, 3, 4,
                binding.AddRmsNormGrads(*got), dtype, "float32", (B, T, D))
    got = torch.autograd.grad(total, (x, res), ds)
    check_grads(_host(r.sum).reshape(-1, D), _host(weight.detach()), r.rstd, None, ds64, lengths, p, 3, 4,
                binding.AddRmsNormGrads(*got, None), dtype, "float32", (B, T, D))
    # leaves: their gradients are tensors of their own
    y, total = chain.add_rms_norm(x, res, None, 1e-5, None, p, 3, 4)
    (y.float().sum() + total.float().square().sum()).backward()
    assert x.grad.data_ptr() != res.grad.data_ptr()
    before = res.grad.clone()
    x.grad.zero_()
    assert torch.equal(res.grad, before)
    # nothing added, nothing dropped: sum is x
    y, total = chain.add_rms_norm(x, None, weight)
    assert torch.equal(total, x)
    got = torch.autograd.grad((y, total), (x, weight), (dy, ds))
    r = binding.lfmmi_add_rms_norm(x.detach(), None, weight.detach())
    check_grads(x64.reshape(-1, D), _host(weight.detach()), r.rstd, dy64, ds64, None, 0.0, 0, 0,
                binding.AddRmsNormGrads(got[0], None, got[1]), dtype, "float32", (B, T, D))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("two", [False, True])
def test_gradient_behind_the_lengths_where_sum_is_x(two, dtype):
    # nothing added, nothing dropped: sum is x, rows behind the lengths too, and so is its gradient
    torch = _torch()
    rng = np.random.default_rng(22)
    lengths, T, D = ([1, 0, 1, 1, 0], 1, 50) if two else ([6, 0, 4], 6, 50)
    B = len(lengths)
    shape = (B, D) if two else (B, T, D)
    x, x64 = _values(rng, shape, dtype)
    dy, dy64 = _values(rng, shape, dtype)
    ds, ds64 = _values(rng, shape, dtype)
    weight = torch.from_numpy(rng.normal(1, 0.3, D).astype(np.float32)).cuda().requires_grad_()
    x.requires_grad_()
    behind = torch.from_numpy(np.arange(T)[None] >= np.array(lengths)[:, None]).cuda().reshape(shape[:-1])
    y, total = chain.add_rms_norm(x, None, weight, 1e-5, lengths)
    assert torch.equal(total, x) and not y[behind].any()
    rstd = binding.lfmmi_add_rms_norm(x.detach(), None, weight.detach(), 1e-5, lengths).rstd
    x64 = np.where(behind.cpu().numpy()[..., None], 0.0, x64)
    for grads, dsum in (((y, total), ds64), ((total,), ds64), ((y,), None)):
        got = torch.autograd.grad(grads, (x, weight), [dy if v is y else ds for v in grads], retain_graph=True, allow_unused=True)
        want = ds[behind] if dsum is not None else torch.zeros_like(ds[behind])
        assert torch.equal(got[0][behind], want)
        inside = got[0].clone()
        inside[behind] = 0
        check_grads(x64.reshape(-1, D), _host(weight.detach()), rstd, dy64 if len(grads) > 1 or dsum is None else None, dsum, lengths, 0.0, 0, 0,
                    binding.AddRmsNormGrads(inside, None, got[1]), dtype, "float32", shape)


def test_gradient_behind_the_lengths_captured():
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((3, 6, 50), generator=gen, device="cuda").requires_grad_()
    weight = torch.ones(50, device="cuda").requires_grad_()
    dy, ds = (torch.randn((3, 6, 50), generator=gen, device="cuda") for _ in range(2))

    def step():
        return torch.autograd.grad(chain.add_rms_norm(x, None, weight, 1e-5, [6, 0, 4]), (x, weight), (dy, ds))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(4):
        dy.copy_(torch.randn_like(dy))
        ds.mul_(-1.5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step()))
        assert torch.equal(out[0][1], ds[1]) and torch.equal(out[0][2, 4:], ds[2, 4:])


@pytest.mark.parametrize("of_x,of_residual", [("bfloat16", "float32"), ("float16", "float32"), ("float32", "bfloat16"), ("bfloat16", "float16")])
def test_a_residual_of_another_type(of_x, of_residual):
    # as torch adds them: in float32, no bit of either is lost
    torch = _torch()
    rng = np.random.default_rng(23)
    B, T, D = 3, 6, 50
    lengths = [6, 0, 4]
    x, x64 = _values(rng, (B, T, D), of_x)
    res, r64 = _values(rng, (B, T, D), of_residual, 3.0)
    for w_dtype in (of_x, "float32"):
        weight = torch.from_numpy(rng.normal(1, 0.3, D).astype(np.float32)).to(getattr(torch, w_dtype)).cuda()
        leaves = [v.detach().requires_grad_() for v in (x, res, weight)]
        for p in (0.0, 0.3):
            y, total = chain.add_rms_norm(*leaves, 1e-5, lengths, p, 3, 4)
            assert y.dtype == total.dtype == torch.float32
            r = binding.lfmmi_add_rms_norm(x.float(), res.float(), weight.float(), 1e-5, lengths, p, 3, 4)
            assert torch.equal(y, r.y) and torch.equal(total, r.sum)
            dy, ds = torch.randn_like(y), torch.randn_like(y)
            got = torch.autograd.grad((y, total), leaves, (dy, ds))
            want = binding.lfmmi_add_rms_norm_backward(r.sum, r.rstd, weight.float(), dy, ds, lengths, p, 3, 4)
            assert all(a.dtype == b.dtype and torch.equal(a, c.to(a.dtype)) for a, b, c in zip(got, leaves, want))


def test_gradients_against_differences():
    # of the kernels' own loss: fp32, a step of 2^-6 and values near 1, so that the difference of two
    # losses of some 100 terms errs by 2 * 100 * 2^-24 * 8 / 2^-5 = 3e-3 at most, and its curvature by 2^-12
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, res = (torch.randn((2, 20), generator=gen, device="cuda", requires_grad=True) for _ in range(2))
    weight = torch.randn(20, generator=gen, device="cuda", requires_grad=True)
    wy, ws = (torch.randn((2, 20), generator=gen, device="cuda") for _ in range(2))

    def loss(a, b, c):
        y, total = chain.add_rms_norm(a, b, c, 1e-2, None, 0.25, 8, 9)
        return (wy * y).double().sum() + (ws * total).double().sum()

    grads = torch.autograd.grad(loss(x, res, weight), (x, res, weight))
    inputs = [x.detach(), res.detach(), weight.detach()]
    for which, grad in enumerate(grads):
        flat = inputs[which].reshape(-1)
        for i in range(0, flat.numel(), 3):
            old, both = float(flat[i]), []
            for sign in (1, -1):
                flat[i] = old + sign * 2.0 ** -6
                both.append(float(loss(*inputs)))
            flat[i] = old
            assert abs((both[0] - both[1]) * 32 - float(grad.reshape(-1)[i])) < 6e-3


def test_norm_captured_and_replayed():
    torch = _torch()
    rng = np.random.default_rng(31)
    B, T, D = 4, 300, 640
    x, _ = _values(rng, (B, T, D), "bfloat16")
    res, _ = _values(rng, (B, T, D), "bfloat16")
    dy, _ = _values(rng, (B, T, D), "bfloat16")
    weight = torch.ones(D, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    kw = dict(lengths=[300, 7, 0, 299], p=0.1, seed=3, offset=5)
    out = binding.lfmmi_add_rms_norm(x, res, weight, step=step, **kw)
    grads = binding.lfmmi_add_rms_norm_backward(out.sum, out.rstd, weight, dy, step=step, **kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.lfmmi_add_rms_norm(x, res, weight, step=step, out=out, **kw)
        binding.lfmmi_add_rms_norm_backward(out.sum, out.rstd, weight, dy, step=step, out=grads, **kw)
    for k in range(4):
        step.fill_(k)
        x.mul_(1.25)
        dy.neg_()
        graph.replay()
        torch.cuda.synchronize()
        want = binding.lfmmi_add_rms_norm(x, res, weight, step=step, **kw)
        want_g = binding.lfmmi_add_rms_norm_backward(want.sum, want.rstd, weight, dy, **dict(kw, offset=5 + k))
        assert all(torch.equal(a, b) for a, b in zip(out[:3], want[:3])) and all(torch.equal(a, b) for a, b in zip(grads, want_g))


def test_rows_beyond_32_bits_of_offset():
    torch = _torch()
    B, D = 70000, 65536
    x = torch.zeros((B, D), dtype=torch.bfloat16, device="cuda")
    x[-1, ::2] = 2.0
    r = binding.lfmmi_add_rms_norm(x)
    assert not r.y[-2].any() and (r.y[-1, ::2].float() - 2.0 ** 0.5).abs().max() < 0.01 and not r.y[-1, 1::2].any()
    y = binding.lfmmi_dropout(x, 0.5, 1, out=x)
    mask = torch.from_numpy(oracle.kept([B - 1], D, 0.5, 1, 0)[0]).cuda()
    assert torch.equal(y[-1, ::2] == 4.0, mask[::2]) and not y[-2].any()
