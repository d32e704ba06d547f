"""Rows of a table for given tokens and the gradient of the table, against the 64-bit forms."""
import numpy as np
import pytest

from paper_2005_09824_amd import binding, chain
from tests import layers_oracle as oracle

pytestmark = pytest.mark.gpu

DTYPES = ["float32", "bfloat16", "float16"]


def _torch():
    import torch
    return torch


def _values(rng, shape, dtype, sigma=1.0):
    """(device tensor, its values in 64 bits)"""
    torch = _torch()
    x = torch.from_numpy(rng.normal(0, sigma, shape).astype(np.float32)).to(getattr(torch, dtype)).cuda()
    return x, x.double().cpu().numpy()


def _live(B, T, lengths):
    live = np.ones((B, T), bool)
    if lengths is not None:
        live &= np.arange(T)[None] < np.asarray(lengths)[:, None]
    return live.reshape(-1)


def _close(got, want, tol, what):
    got = got.double().cpu().numpy().reshape(want.shape)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), what
    off, tol = np.abs(got - want)[~nan], np.broadcast_to(tol, want.shape)[~nan]
    assert np.all(off <= tol), (what, off.max(), (off / np.maximum(tol, 1e-300)).max())


def _check_forward(table, table64, tokens, lengths, scale, r):
    t = tokens.cpu().numpy().astype(np.int64)
    B, T = t.shape if t.ndim == 2 else (t.shape[0], 1)
    want, status = oracle.embed(table64, t.reshape(-1), _live(B, T, lengths), float(np.float32(scale)))
    dtype = str(table.dtype).replace("torch.", "")
    tol = np.abs(want) * (oracle.U + oracle.rounding(dtype)) + oracle.TINY[dtype]
    _close(r[0], want, np.where(np.isnan(tol), 0.0, tol), "rows")
    assert np.array_equal(r[1].cpu().numpy().reshape(-1), status)


def _check_backward(g64, dtype, tokens, lengths, scale, grad, old=None, accumulate=False):
    t = tokens.cpu().numpy().astype(np.int64)
    B, T = t.shape if t.ndim == 2 else (t.shape[0], 1)
    V, D = grad.shape
    want, size, count = oracle.embed_grad(g64.reshape(-1, D), t.reshape(-1), _live(B, T, lengths),
                                          float(np.float32(scale)), V)
    if accumulate:
        want = want + old
    tol = oracle.bound_embed_grad(want, size, count, dtype, old if accumulate else None)
    none = count == 0
    tol[none] = 0.0   # zeros, or left as they are
    _close(grad, want, tol, "gradient")


SHAPES = [(1, 1, 1, 1), (3, 2, 5, 7), (1, 1, 4096, 64), (17, 9, 10, 63), (2, 700, 84, 64), (5, 333, 3, 65), (300, 3, 50, 40),
          (1, 5000, 1000, 17), (64, 33, 1025, 128), (4, 1000, 40000, 24), (1, 3, 200000, 8), (2, 90, 7, 2049), (1, 40, 3, 8200),
          (1, 70, 2, 4097), (2, 2049, 1, 8),
          (1, 2047, 600, 8), (2, 1024, 2048, 9), (1, 500, 2049, 16), (1, 1030, 90, 24), (1, 2048, 300000, 8), (1, 140000, 70, 8),
          (600, 4, 33, 16)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,T,V,D", SHAPES)
def test_rows_and_gradients(B, T, V, D, dtype):
    torch = _torch()
    rng = np.random.default_rng(B * 7 + T * 3 + V + D)
    table, table64 = _values(rng, (V, D), dtype)
    tokens = torch.from_numpy(rng.integers(-1 if V > 1 else 0, V + (1 if V > 5 else 0), (B, T))).cuda()
    lengths = rng.integers(0, T + 1, B).astype(np.int32)
    g, g64 = _values(rng, (B, T, D), dtype)
    for lens, scale in ((None, 1.0), (lengths, 1.7)):
        _check_forward(table, table64, tokens, lens, scale, binding.lfmmi_embed_tokens(table, tokens, lens, scale))
        grad = binding.lfmmi_embed_tokens_backward(g, tokens, V, lens, scale)
        _check_backward(g64, dtype, tokens, lens, scale, grad)
        again = binding.lfmmi_embed_tokens_backward(g, tokens.to(torch.int32), V, lens, scale)
        assert torch.equal(again, grad)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [2, 300, 70000, (1 << 20) + 3])
def test_frequent_tokens(V, dtype):
    # half of all positions one token, a tenth another, one token alone at the very end
    torch = _torch()
    rng = np.random.default_rng(V)
    N, D = 9001, 24
    t = rng.integers(0, V, N)
    t[rng.random(N) < 0.5] = V // 2
    t[rng.random(N) < 0.1] = 0
    t[-1] = V - 1
    tokens = torch.from_numpy(t).cuda()
    g, g64 = _values(rng, (N, D), dtype)
    grad = binding.lfmmi_embed_tokens_backward(g, tokens, V)
    _check_backward(g64, dtype, tokens, None, 1.0, grad)
    for _ in range(3):   # pieces of frequent tokens are handed out by chance; the sums do not show it
        assert torch.equal(binding.lfmmi_embed_tokens_backward(g, tokens, V), grad)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_one_token_of_most_positions(dtype):
    # half a million positions of one token, all of one gradient, so that the roundings of a running sum add up. A value goes
    # through 15 additions of its piece of 16 and 3 of eight pieces; the sum of a wave's 1,025 eights, which keeps what it loses,
    # errs by one step and (1,025 U)^2 < 1 of them; 4 additions of positions behind the pieces, 3 of the waves' sums, the
    # scale: 28, and 2 for these steps' own products
    torch = _torch()
    N, V, D = (1 << 19) + 37, 3, 24
    tokens = torch.ones(N, dtype=torch.int64, device="cuda")
    tokens[[5, 4000, N - 1]] = torch.tensor([0, 2, 0], device="cuda")
    row = torch.linspace(-0.3, 0.3, D, device="cuda").to(getattr(torch, dtype))
    grad = binding.lfmmi_embed_tokens_backward(row.expand(N, D), tokens, V)
    want = row.double().cpu().numpy()[None] * np.array([[2.0], [N - 3.0], [1.0]])
    tol = np.abs(want) * (30 * oracle.U + oracle.rounding(dtype)) + oracle.TINY[dtype]
    assert np.all(np.abs(grad.double().cpu().numpy() - want) <= tol), (np.abs(grad.double().cpu().numpy() - want) / tol).max()
    # a sum beyond the type is the infinity it would be in any order, and a NaN stays one
    row = torch.tensor([1e38, -1e38, float("inf"), float("nan")], device="cuda")
    grad = binding.lfmmi_embed_tokens_backward(row.expand(N, 4), tokens, V)[1].tolist()
    assert grad[:3] == [np.inf, -np.inf, np.inf] and np.isnan(grad[3])


@pytest.mark.parametrize("count", [15, 16, 17, 31, 32, 33, 63, 64, 65, 95, 96, 97, 2047, 2048, 2049, 4097])
def test_counts_next_to_a_piece(count):
    torch = _torch()
    rng = np.random.default_rng(count)
    tokens = torch.from_numpy(np.concatenate([np.full(count, 3), np.full(5, 1), np.full(count, 4)])).cuda()
    g, g64 = _values(rng, (len(tokens), 70), "float32")
    grad = binding.lfmmi_embed_tokens_backward(g, tokens, 6)
    _check_backward(g64, "float32", tokens, None, 1.0, grad)


@pytest.mark.parametrize("dtype", DTYPES)
def test_accumulating_leaves_other_rows_alone(dtype):
    torch = _torch()
    rng = np.random.default_rng(5)
    V, D, N = 400, 31, 3000
    t = rng.integers(0, 90, N)
    t[:1000] = 7
    t[5] = -4
    tokens = torch.from_numpy(t).cuda()
    g, g64 = _values(rng, (N, D), dtype)
    grad, old = _values(rng, (V, D), dtype)
    version = grad._version
    r = binding.lfmmi_embed_tokens_backward(g, tokens, V, scale=0.5, grad=grad, accumulate=True)
    assert r is grad and grad._version > version
    _check_backward(g64, dtype, tokens, None, 0.5, grad, old, True)


def test_all_rows_ignored_and_no_rows():
    torch = _torch()
    g = torch.full((4, 6, 10), float("nan"), device="cuda")
    tokens = torch.tensor([[-1, 99, 5, 5, 5, 5]] * 4, device="cuda")
    grad = binding.lfmmi_embed_tokens_backward(g, tokens, 20, [2, 2, 1, 0])
    assert not grad.any()   # what is not read is not added, whatever it holds
    rows, status = binding.lfmmi_embed_tokens(torch.ones((20, 10), device="cuda"), tokens, [2, 2, 1, 0])
    assert torch.isnan(rows[:2, 1]).all() and not rows[:2, 0].any() and not rows[:, 2:].any() and not rows[2:].any()
    assert status.tolist() == [[0, 4, 0, 0, 0, 0]] * 2 + [[0] * 6] * 2
    for shape in ((0, 6), (4, 0)):
        none = torch.zeros(shape, dtype=torch.int64, device="cuda")
        assert not binding.lfmmi_embed_tokens_backward(torch.zeros(shape + (10,), device="cuda"), none, 20).any()
        assert binding.lfmmi_embed_tokens(torch.ones((20, 10), device="cuda"), none)[0].shape == shape + (10,)


@pytest.mark.parametrize("dtype", DTYPES)
def test_views(dtype):
    # rows of a table and of gradients that start anywhere; what lies around them is NaN
    torch = _torch()
    rng = np.random.default_rng(8)
    V, D, B, T = 50, 37, 3, 11
    base = torch.full((V, D + 9), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    table = base[:, 5:5 + D]
    table.copy_(torch.from_numpy(rng.normal(0, 1, (V, D)).astype(np.float32)))
    tokens = torch.from_numpy(rng.integers(0, V, (B, T))).cuda()
    _check_forward(table, table.double().cpu().numpy(), tokens, None, 2.0, binding.lfmmi_embed_tokens(table, tokens, scale=2.0))
    wide = torch.full((B, T + 2, D + 3), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    g = wide[:, 1:T + 1, 3:]
    g.copy_(torch.from_numpy(rng.normal(0, 1, (B, T, D)).astype(np.float32)))
    _check_backward(g.double().cpu().numpy(), dtype, tokens, None, 1.0, binding.lfmmi_embed_tokens_backward(g, tokens, V))
    same = table[:1].expand(4, D)   # one row for all tokens
    rows, _status = binding.lfmmi_embed_tokens(same, tokens.clamp(max=3))
    assert torch.equal(rows, table[0].expand(B, T, D))
    one = g[:1, :1].expand(B, T, D)   # the gradient of a sum
    _check_backward(one.double().cpu().numpy(), dtype, tokens, None, 1.0, binding.lfmmi_embed_tokens_backward(one, tokens, V))


def test_outputs_that_are_passed_in():
    torch = _torch()
    table = torch.randn((30, 12), device="cuda")
    tokens = torch.tensor([3, -1, 30], device="cuda")
    out, status = torch.full((3, 12), 7.0, device="cuda"), torch.full((3,), 9, dtype=torch.int32, device="cuda")
    version = out._version
    r = binding.lfmmi_embed_tokens(table, tokens, out=out, status=status)
    assert r[0] is out and r[1] is status and out._version > version
    assert torch.equal(out[0], table[3]) and not out[1].any() and torch.isnan(out[2]).all() and status.tolist() == [0, 0, 4]
    for kw in (dict(out=out[:2]), dict(out=out.double()), dict(status=out), dict(out=torch.zeros((3, 24), device="cuda")[:, ::2])):
        with pytest.raises(ValueError):
            binding.lfmmi_embed_tokens(table, tokens, **kw)
    with pytest.raises(binding.LfmmiError):
        binding.lfmmi_embed_tokens(table, tokens, out=table[:3])


@pytest.mark.parametrize("dtype", DTYPES)
def test_through_autograd(dtype):
    torch = _torch()
    rng = np.random.default_rng(11)
    V, D, B, T = 40, 20, 3, 50
    table, table64 = _values(rng, (V, D), dtype)
    table.requires_grad_()
    tokens = torch.from_numpy(rng.integers(-1, V, (B, T))).cuda()
    lengths = [50, 20, 0]
    rows, status = chain.embed_tokens(table, tokens, lengths, 3.0)
    g, g64 = _values(rng, (B, T, D), dtype)
    lengths[0] = 1   # (the call has a copy)
    (grad,) = torch.autograd.grad(rows, table, g)
    _check_forward(table.detach(), table64, tokens, [50, 20, 0], 3.0, (rows.detach(), status))
    _check_backward(g64, dtype, tokens, [50, 20, 0], 3.0, grad)
    # a sum's gradient is one value for all
    (grad,) = torch.autograd.grad(chain.embed_tokens(table, tokens)[0].sum(), table)
    counts = torch.bincount(tokens[tokens >= 0], minlength=V)
    assert torch.equal(grad, counts.to(grad.dtype).unsqueeze(1).expand(V, D))


def test_captured_and_replayed():
    torch = _torch()
    rng = np.random.default_rng(12)
    V, D, B, T = 500, 64, 4, 900
    table, _ = _values(rng, (V, D), "float32")
    g, _ = _values(rng, (B, T, D), "float32")
    tokens = torch.from_numpy(rng.integers(0, V, (B, T))).cuda()
    tokens[:, :300] = 9
    out = (torch.empty((B, T, D), device="cuda"), torch.empty((B, T), dtype=torch.int32, device="cuda"))
    grad = torch.empty((V, D), device="cuda")

    def step():
        binding.lfmmi_embed_tokens(table, tokens, out=out[0], status=out[1])
        binding.lfmmi_embed_tokens_backward(g, tokens, V, grad=grad)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        tokens.copy_(torch.from_numpy(rng.integers(-1, V, (B, T))))
        if k % 2:
            tokens[:, 100:600] = k
        g.mul_(1.1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], binding.lfmmi_embed_tokens(table, tokens)[0])
        assert torch.equal(grad, binding.lfmmi_embed_tokens_backward(g, tokens, V))


def test_on_another_stream():
    torch = _torch()
    rng = np.random.default_rng(13)
    table, table64 = _values(rng, (100, 32), "float32")
    tokens = torch.from_numpy(rng.integers(0, 100, 4000)).cuda()
    g, g64 = _values(rng, (4000, 32), "float32")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rows = binding.lfmmi_embed_tokens(table, tokens, stream=side.cuda_stream)
    grad = binding.lfmmi_embed_tokens_backward(g, tokens, 100, stream=side.cuda_stream)
    side.synchronize()
    _check_forward(table, table64, tokens, None, 1.0, rows)
    _check_backward(g64, "float32", tokens, None, 1.0, grad)


def test_offsets_beyond_32_bits():
    # a table of 5 GB and gradients whose rows are 2^32 values apart in all
    torch = _torch()
    V, D = 40000, 65536
    table = torch.empty((V, D), dtype=torch.bfloat16, device="cuda")
    table[-1] = 3.0
    table[V - 2] = 5.0
    tokens = torch.tensor([V - 1, V - 2], device="cuda")
    rows, _status = binding.lfmmi_embed_tokens(table, tokens)
    assert (rows[0] == 3).all() and (rows[1] == 5).all()
    g = torch.ones((2, D), dtype=torch.bfloat16, device="cuda")
    grad = binding.lfmmi_embed_tokens_backward(g, tokens, V, grad=table)
    assert (grad[-2:] == 1).all() and not grad[:-2].any()
    del table, grad
    big = torch.empty((70000, 65536), dtype=torch.bfloat16, device="cuda")
    big[69999] = 2.0
    tokens = torch.full((70000,), -1, device="cuda")
    tokens[69999] = 1
    grad = binding.lfmmi_embed_tokens_backward(big, tokens, 2)
    assert (grad[1] == 2).all() and not grad[0].any()
