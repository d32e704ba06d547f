"""What the operators around an output layer refuse before they touch a GPU, and the 64-bit forms
that their kernels are compared with."""
import ctypes

import numpy as np
import pytest

from paper_2005_09824_amd import binding, chain
from tests import layers_oracle as oracle

INVALID, UNSUPPORTED = 1, 5
P = 1 << 16   # an aligned address that nothing reads: every call here is refused
FAR = 1 << 40


def _refused(code, want, text):
    assert code == want and text in binding.lfmmi_last_error(), (code, binding.lfmmi_last_error())


def _lens(v):
    return None if v is None else np.asarray(v, np.int32)


def _embed(lengths=None, **kw):
    a = dict(table=P, dtype=0, V=10, D=4, stride=4, tokens=2 * P, token_bytes=8, B=2, T=3, scale=1.0, out=3 * P,
             status=4 * P)
    a.update(kw)
    lens = _lens(lengths)
    return binding.load_library().lfmmi_embed_tokens(
        a["table"], a["dtype"], a["V"], a["D"], a["stride"], a["tokens"], a["token_bytes"], a["B"], a["T"],
        None if lens is None else lens.ctypes.data, a["scale"], a["out"], a["status"], None)


def _embed_backward(lengths=None, **kw):
    a = dict(g=P, dtype=0, V=10, D=4, stride_b=12, stride_t=4, tokens=2 * P, token_bytes=8, B=2, T=3, scale=1.0,
             accumulate=0, grad=3 * P, ws=FAR, size=1 << 20)
    a.update(kw)
    lens = _lens(lengths)
    return binding.load_library().lfmmi_embed_tokens_backward(
        a["g"], a["dtype"], a["V"], a["D"], a["stride_b"], a["stride_t"], a["tokens"], a["token_bytes"], a["B"],
        a["T"], None if lens is None else lens.ctypes.data, a["scale"], a["accumulate"], a["grad"], a["ws"],
        a["size"], None)


TOKEN_CALLS = [
    (dict(dtype=3), INVALID, "dtype"), (dict(V=0), INVALID, "V"), (dict(D=0), INVALID, "D"),
    (dict(D=(1 << 24) + 1), UNSUPPORTED, "D"), (dict(B=-1), INVALID, "B and T"), (dict(T=-1), INVALID, "B and T"),
    (dict(B=1 << 16, T=1 << 15), UNSUPPORTED, "B * T"), (dict(scale=0.0), INVALID, "scale"),
    (dict(scale=float("nan")), INVALID, "scale"), (dict(scale=-1.0), INVALID, "scale"),
    (dict(token_bytes=2), INVALID, "token_bytes"), (dict(tokens=None), INVALID, "null"),
    (dict(tokens=2 * P + 4), INVALID, "aligned"), (dict(lengths=[3, 4]), INVALID, "lengths[1]"),
    (dict(lengths=[-1, 0]), INVALID, "lengths[0]"),
]


@pytest.mark.parametrize("kw,code,text", TOKEN_CALLS + [
    (dict(stride=-1), INVALID, "strides"), (dict(stride=1 << 60), UNSUPPORTED, "strides"),
    (dict(table=None), INVALID, "null"), (dict(out=None), INVALID, "null"), (dict(table=P + 2), INVALID, "aligned"),
    (dict(out=3 * P + 1), INVALID, "aligned"), (dict(status=4 * P + 2), INVALID, "aligned"),
    (dict(out=P + 36 * 4), INVALID, "overlaps"), (dict(out=2 * P), INVALID, "overlaps"),
    (dict(status=3 * P + 92), INVALID, "overlaps"), (dict(stride=20, out=P + 180 * 4), INVALID, "overlaps"),
])
def test_refused_embeddings(kw, code, text):
    _refused(_embed(**kw), code, text)


@pytest.mark.parametrize("kw,code,text", TOKEN_CALLS + [
    (dict(stride_b=-1), INVALID, "strides"), (dict(stride_t=1 << 60), UNSUPPORTED, "strides"),
    (dict(g=None), INVALID, "null"), (dict(grad=None), INVALID, "null"), (dict(ws=None), INVALID, "workspace"),
    (dict(ws=FAR + 8), INVALID, "workspace"), (dict(size=8), INVALID, "workspace"),
    (dict(grad=P), INVALID, "overlaps"), (dict(grad=2 * P + 40), INVALID, "overlaps"),
    (dict(grad=FAR), INVALID, "overlaps"), (dict(ws=P - 16), INVALID, "overlaps"), (dict(g=P + 1), INVALID, "aligned"),
])
def test_refused_gradients_of_embeddings(kw, code, text):
    _refused(_embed_backward(**kw), code, text)


def test_embedding_calls_with_nothing_to_do():
    assert _embed(B=0) == 0 and _embed(T=0, table=None) == 0
    assert _embed_backward(B=0, accumulate=1, g=None, tokens=None) == 0


def _dropout(**kw):
    a = dict(x=P, dtype=0, R=3, D=5, stride=5, p=0.1, seed=1, offset=2, step=None, y=2 * P)
    a.update(kw)
    return binding.load_library().lfmmi_dropout(a["x"], a["dtype"], a["R"], a["D"], a["stride"], a["p"], a["seed"],
                                                a["offset"], a["step"], a["y"], None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dtype=-1), INVALID, "dtype"), (dict(R=-1), INVALID, "R and D"), (dict(D=-1), INVALID, "R and D"),
    (dict(stride=-1), INVALID, "strides"), (dict(stride=1 << 60), UNSUPPORTED, "strides"),
    (dict(p=-0.1), INVALID, "p outside"), (dict(p=1.1), INVALID, "p outside"), (dict(p=float("nan")), INVALID, "p outside"),
    (dict(x=None), INVALID, "null"), (dict(y=None), INVALID, "null"), (dict(x=P + 2), INVALID, "aligned"),
    (dict(y=2 * P + 1), INVALID, "aligned"), (dict(step=P + 4), INVALID, "aligned"), (dict(y=P + 4), INVALID, "overlaps"),
    (dict(y=P - 56), INVALID, "overlaps"), (dict(x=P, y=P, stride=4), INVALID, "overlap"), (dict(step=2 * P + 56), INVALID, "overlaps"),
    (dict(x=P, y=P, step=P + 8), INVALID, "overlaps"),
])
def test_refused_dropout(kw, code, text):
    _refused(_dropout(**kw), code, text)


def test_dropout_of_nothing():
    assert _dropout(R=0, x=None, y=None) == 0 and _dropout(D=0, x=None, y=None) == 0


def _norm(lengths=None, **kw):
    a = dict(x=P, stride_b=12, stride_t=4, residual=2 * P, rb=12, rt=4, dtype=0, B=2, T=3, D=4, weight=3 * P, wd=0,
             eps=1e-6, p=0.1, seed=0, offset=0, step=None, sum=4 * P, y=5 * P, rstd=6 * P, q=7 * P, q_scale=8 * P)
    a.update(kw)
    lens = _lens(lengths)
    return binding.load_library().lfmmi_add_rms_norm(
        a["x"], a["stride_b"], a["stride_t"], a["residual"], a["rb"], a["rt"], a["dtype"], a["B"], a["T"], a["D"],
        None if lens is None else lens.ctypes.data, a["weight"], a["wd"], a["eps"], a["p"], a["seed"], a["offset"],
        a["step"], a["sum"], a["y"], a["rstd"], a["q"], a["q_scale"], None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dtype=4), INVALID, "dtype"), (dict(wd=1), INVALID, "weight_dtype"), (dict(D=0), INVALID, "D"),
    (dict(D=(1 << 24) + 1), UNSUPPORTED, "D"), (dict(B=-1), INVALID, "B and T"), (dict(B=1 << 16, T=1 << 15), UNSUPPORTED, "B * T"),
    (dict(stride_b=-1), INVALID, "strides"), (dict(rt=-1), INVALID, "strides"), (dict(rb=1 << 60), UNSUPPORTED, "strides"),
    (dict(eps=0.0), INVALID, "eps"), (dict(eps=-1.0), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"),
    (dict(eps=float("inf")), INVALID, "eps"), (dict(p=2.0), INVALID, "p outside"), (dict(x=None), INVALID, "x is null"),
    (dict(sum=None), INVALID, "sum is null"), (dict(sum=None, residual=None), INVALID, "sum is null"),
    (dict(q=None), INVALID, "go together"), (dict(q_scale=None), INVALID, "go together"),
    (dict(x=P + 2), INVALID, "aligned"), (dict(residual=2 * P + 1), INVALID, "aligned"), (dict(weight=3 * P + 2), INVALID, "aligned"),
    (dict(rstd=6 * P + 1), INVALID, "aligned"), (dict(y=P), INVALID, "overlaps"), (dict(y=4 * P + 92), INVALID, "overlaps"),
    (dict(q=3 * P), INVALID, "overlaps"), (dict(sum=P + 4), INVALID, "overlaps"), (dict(sum=P, stride_t=5, stride_b=15), INVALID, "overlaps"),
    (dict(sum=2 * P, rb=0), INVALID, "overlaps"), (dict(sum=P, residual=P, rb=0), INVALID, "overlaps"),
    (dict(lengths=[4, 0]), INVALID, "lengths[0]"), (dict(rstd=3 * P), INVALID, "overlaps"),
])
def test_refused_norms(kw, code, text):
    _refused(_norm(**kw), code, text)


@pytest.mark.parametrize("eps", [0.9e-30, 1.1e20, 1e30, 3e38])
def test_eps_beyond_what_sums_of_squares_leave_room_for_is_refused(eps):
    _refused(_norm(eps=eps), INVALID, "eps")


def _norm_backward(lengths=None, **kw):
    a = dict(sum=P, stride_b=12, stride_t=4, dtype=0, B=2, T=3, D=4, weight=2 * P, wd=0, rstd=3 * P, dy=4 * P, ds=5 * P,
             p=0.1, seed=0, offset=0, step=None, dx=6 * P, dr=7 * P, dw=8 * P, ws=FAR, size=1 << 20)
    a.update(kw)
    lens = _lens(lengths)
    return binding.load_library().lfmmi_add_rms_norm_backward(
        a["sum"], a["stride_b"], a["stride_t"], a["dtype"], a["B"], a["T"], a["D"],
        None if lens is None else lens.ctypes.data, a["weight"], a["wd"], a["rstd"], a["dy"], a["ds"], a["p"], a["seed"],
        a["offset"], a["step"], a["dx"], a["dr"], a["dw"], a["ws"], a["size"], None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dtype=4), INVALID, "dtype"), (dict(wd=2), INVALID, "weight_dtype"), (dict(weight=None, wd=7), INVALID, "weight_dtype"),
    (dict(D=0), INVALID, "D"), (dict(T=-1), INVALID, "B and T"), (dict(stride_t=-1), INVALID, "strides"), (dict(p=-1.0), INVALID, "p outside"),
    (dict(sum=None), INVALID, "null"), (dict(rstd=None), INVALID, "null"), (dict(dy=None, ds=None), INVALID, "grad_y"),
    (dict(sum=P + 1), INVALID, "aligned"), (dict(dw=8 * P + 2), INVALID, "aligned"), (dict(ws=None), INVALID, "workspace"),
    (dict(ws=FAR + 4), INVALID, "workspace"), (dict(size=8), INVALID, "workspace"), (dict(dx=7 * P), INVALID, "overlaps"),
    (dict(dx=P), INVALID, "overlaps"), (dict(dr=4 * P + 4), INVALID, "overlaps"), (dict(dw=3 * P), INVALID, "overlaps"),
    (dict(ws=5 * P), INVALID, "overlaps"), (dict(lengths=[3, -1]), INVALID, "lengths[1]"),
])
def test_refused_gradients_of_norms(kw, code, text):
    _refused(_norm_backward(**kw), code, text)


def _verify(lengths=None, **kw):
    a = dict(x=P, dtype=0, B=2, K=3, V=10, stride_b=40, stride_t=10, draft=2 * P, db=30, dt=10, drafted=3 * P, token_bytes=8,
             scale=1.0, draft_scale=1.0, u=4 * P, accepted=5 * P, tokens=6 * P, status=7 * P, ws=FAR, size=1 << 20)
    a.update(kw)
    lens = _lens(lengths)
    return binding.load_library().lfmmi_verify_tokens(
        a["x"], a["dtype"], a["B"], a["K"], a["V"], a["stride_b"], a["stride_t"], a["draft"], a["db"], a["dt"], a["drafted"],
        a["token_bytes"], None if lens is None else lens.ctypes.data, a["scale"], a["draft_scale"], a["u"], a["accepted"],
        a["tokens"], a["status"], a["ws"], a["size"], None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dtype=3), INVALID, "dtype"), (dict(B=-1), INVALID, "B and K"), (dict(K=-1), INVALID, "B and K"), (dict(V=0), INVALID, "V"),
    (dict(V=(1 << 30) + 1), UNSUPPORTED, "V"), (dict(B=1 << 16, K=1 << 14), UNSUPPORTED, "2 K + 1"),
    (dict(B=0, K=(1 << 31) - 1), UNSUPPORTED, "2 K + 1"), (dict(stride_b=-1), INVALID, "strides"), (dict(dt=-1), INVALID, "strides"),
    (dict(stride_t=1 << 60), UNSUPPORTED, "strides"), (dict(scale=0.0), INVALID, "scale"), (dict(draft_scale=1e7), INVALID, "scale"),
    (dict(lengths=[4, 0]), INVALID, "lengths[0]"), (dict(token_bytes=1), INVALID, "token_bytes"), (dict(u=None), INVALID, "uniforms"),
    (dict(x=None), INVALID, "null"), (dict(drafted=None), INVALID, "null"), (dict(accepted=None), INVALID, "null"),
    (dict(tokens=None), INVALID, "null"), (dict(x=P + 2), INVALID, "aligned"), (dict(drafted=3 * P + 4), INVALID, "aligned"),
    (dict(u=4 * P + 2), INVALID, "aligned"), (dict(ws=None), INVALID, "workspace"), (dict(ws=FAR + 1), INVALID, "workspace"),
    (dict(size=16), INVALID, "workspace"), (dict(tokens=P), INVALID, "overlaps"), (dict(accepted=6 * P + 28), INVALID, "overlaps"),
    (dict(ws=2 * P), INVALID, "overlaps"), (dict(status=4 * P), INVALID, "overlaps"),
])
def test_refused_verifications(kw, code, text):
    _refused(_verify(**kw), code, text)


def test_verification_of_no_sequence():
    assert _verify(B=0) == 0


def test_workspaces():
    lib = binding.load_library()
    n = ctypes.c_int64(-1)
    for name, good, bad in (("lfmmi_embed_tokens_workspace", (10, 4, 2, 3), [(0, 4, 2, 3), (10, 0, 2, 3), (10, 4, -1, 3)]),
                            ("lfmmi_add_rms_norm_workspace", (2, 3, 4), [(-1, 3, 4), (2, -3, 4), (2, 3, 0)]),
                            ("lfmmi_verify_tokens_workspace", (2, 3, 10), [(-1, 3, 10), (2, -1, 10), (2, 3, 0)])):
        call = getattr(lib, name)
        assert call(*good, ctypes.byref(n)) == 0 and n.value > 0
        assert call(*good, None) == INVALID
        for args in bad:
            assert call(*args, ctypes.byref(n)) == INVALID
    assert lib.lfmmi_embed_tokens_workspace(10, (1 << 24) + 1, 2, 3, ctypes.byref(n)) == UNSUPPORTED
    assert lib.lfmmi_embed_tokens_workspace(10, 4, 1 << 16, 1 << 15, ctypes.byref(n)) == UNSUPPORTED
    # (the partial sums of the largest call that is taken pass 2^32 bytes, not 2^63)
    assert lib.lfmmi_embed_tokens_workspace((1 << 31) - 1, 1 << 24, (1 << 31) - 1, 1, ctypes.byref(n)) == 0 and n.value > 1 << 40


def test_binding_refuses_what_is_not_on_a_gpu():
    import torch
    x, t = torch.zeros((3, 5)), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: binding.lfmmi_embed_tokens(x, t), lambda: binding.lfmmi_embed_tokens_backward(x, t, 4),
                 lambda: binding.lfmmi_dropout(x, 0.1, 0), lambda: binding.lfmmi_add_rms_norm(x),
                 lambda: binding.lfmmi_add_rms_norm_backward(x, x[:, 0], None, x), lambda: binding.lfmmi_verify_tokens(x[None]),
                 lambda: chain.embed_tokens(x, t), lambda: chain.dropout(x, 0.1, 0), lambda: chain.add_rms_norm(x)):
        with pytest.raises(ValueError):
            call()


class _OnGpu:
    """What the binding asks of a tensor of `shape` on a GPU."""
    is_cuda = True

    def __init__(self, shape):
        import torch
        t = torch.empty(1, dtype=torch.float32).expand(shape)
        self.dtype, self.shape, self.device = t.dtype, t.shape, t.device
        self.dim, self.stride = t.dim, lambda: t.stride()[:-1] + (1,)


@pytest.mark.parametrize("shape", [((1 << 32) + 5, 4), (1 << 31, 4), (3, (1 << 32) + 7), ((1 << 32) + 1, 2, 4), (2, 3, 1 << 33)])
def test_sizes_beyond_the_libraries_types_are_refused(shape):
    with pytest.raises(ValueError, match="too many rows or columns"):
        binding._batch_rows(_OnGpu(shape), "x")
    assert binding._batch_rows(_OnGpu((5, 3, 4)), "x")[:4] == (0, 5, 3, 4)


def test_rows_of_any_number_of_dimensions():
    import torch
    x = torch.zeros((4, 6, 5))
    assert binding._flat_rows(x) == (24, 5, 5) and binding._flat_rows(x[:, :, :3]) == (24, 3, 5)
    assert binding._flat_rows(x[1:3, :1]) == (2, 5, 30) and binding._flat_rows(torch.zeros(7)) == (1, 7, 7)
    assert binding._flat_rows(x[0, 0].expand(4, 3, 5)) == (12, 5, 0) and binding._flat_rows(x[:1, :1]) == (1, 5, 5)
    assert binding._flat_rows(torch.zeros(())) == (1, 1, 1)
    for bad in (x[:, :3], x.transpose(0, 1), x.transpose(1, 2), x[:, :, ::2]):
        with pytest.raises(ValueError):
            binding._flat_rows(bad)


# ---- the oracle itself

def test_philox_against_its_authors_vectors():
    # counter, key, result: the known answers published with the generator
    full = 0xFFFFFFFF
    for counter, key, want in (
            ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            ((full,) * 4, (full, full), (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
             (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        assert tuple(oracle.philox(counter, key)) == want
    draw, seed = (3 << 32) + 9, (7 << 40) + 123
    got = oracle.words(np.arange(5)[None], np.array([0, 4, 1 << 31])[:, None], draw, seed)
    for i, r in enumerate((0, 4, 1 << 31)):
        for c in range(5):
            assert got[i, c].tolist() == oracle.philox((c, r, draw & full, draw >> 32), (seed & full, seed >> 32))


def test_oracle_gradients_of_a_norm_against_differences():
    rng = np.random.default_rng(1)
    N, D, p = 3, 5, 0.3
    x, r, w = rng.normal(0, 1, (N, D)), rng.normal(0, 2, (N, D)), rng.normal(1, 0.2, D)
    wy, ws = rng.normal(0, 1, (N, D)), rng.normal(0, 1, (N, D))
    mask = oracle.kept(np.arange(N), D, p, 5, 6)
    total = r + oracle.dropped(x, mask, p)
    d, dw = oracle.norm_grads(total, oracle.norm(total, w, 1e-3)[1], w, wy, ws)
    dx = oracle.dropped(d, mask, p)

    def diff(at, e):
        out = []
        for sign in (1, -1):
            args = [x, r, w]
            args[at] = args[at] + sign * e
            out.append(oracle.norm_loss(args[0], args[1], args[2], 1e-3, mask, p, wy, ws))
        return (out[0] - out[1]) / 2e-6

    for n in range(N):
        for i in range(D):
            e = np.zeros((N, D))
            e[n, i] = 1e-6
            assert abs(diff(0, e) - dx[n, i]) < 1e-7 and abs(diff(1, e) - d[n, i]) < 1e-7
    for i in range(D):
        e = np.zeros(D)
        e[i] = 1e-6
        assert abs(diff(2, e) - dw[i]) < 1e-7


def test_oracle_gradient_of_a_table_against_differences():
    rng = np.random.default_rng(2)
    table, tokens, g = rng.normal(0, 1, (6, 3)), np.array([4, 0, -1, 4, 9, 2]), rng.normal(0, 1, (6, 3))
    live = np.array([1, 1, 1, 1, 1, 0], bool)
    grad = oracle.embed_grad(g, tokens, live, 1.5, 6)[0]
    loss = lambda t: np.nansum(oracle.embed(t, tokens, live, 1.5)[0] * g)
    for v in range(6):
        for i in range(3):
            e = np.zeros_like(table)
            e[v, i] = 1e-6
            assert abs((loss(table + e) - loss(table - e)) / 2e-6 - grad[v, i]) < 1e-8


def test_oracle_of_drafted_tokens_by_hand():
    two = np.log([[0.5, 0.25, 0.25], [0.2, 0.3, 0.5]])
    q = np.log([[0.25, 0.5, 0.25]])
    # u q < p: 0.5 * 0.5 < 0.25 is not; what is left of p - q is token 0
    assert oracle.verify(two, [1], 1, 1.0, [0.5, 0.9], q) == (0, 0, 0)
    assert oracle.verify(two, [1], 1, 1.0, [0.49, 0.21], q) == (1, 1, 0)
    assert oracle.verify(two, [1], 0, 1.0, [0.49, 0.51], q) == (0, 1, 0)
    assert oracle.verify(two, [0], 1, 1.0) == (1, 2, 0) and oracle.verify(two, [2], 1, 1.0) == (0, 0, 0)
    # without the draft's logits: p without the drafted token
    assert oracle.verify(two, [0], 1, 1.0, [0.6, 0.49]) == (0, 1, 0)
    assert oracle.verify(two, [7], 1, 1.0, [0.6, 0.49]) == (0, -1, 4)


def test_oracle_draws_as_the_target_says():
    # whatever the draft says, the first token that comes out is distributed as the target's row
    rng = np.random.default_rng(3)
    x, y = rng.normal(0, 1.5, (2, 6)), rng.normal(0, 1.5, (1, 6))
    p, q = oracle.softmax(x[0], 1.0)[0], oracle.softmax(y[0], 1.0)[0]
    first, u = 0.0, np.linspace(0, 1, 2001)[:-1] + 0.00025
    for d in range(6):
        rows = [oracle.verify(x, [d], 1, 1.0, [a, 0.5], y) for a in u]
        first += q[d] * np.mean([r[0] == 1 for r in rows])
        assert abs(np.mean([r[0] == 1 for r in rows]) - min(1.0, p[d] / q[d])) < 1e-3
    rest = np.maximum(p - q, 0)
    drawn = np.bincount([oracle.draw(rest, a) for a in u], minlength=6) / len(u)
    assert np.abs(drawn - rest / rest.sum()).max() < 1e-3 and abs(first - np.minimum(p, q).sum()) < 1e-3
