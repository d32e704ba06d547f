"""Drafted tokens against the target's logits, against the 64-bit form: whole numbers, equal."""
import numpy as np
import pytest

from paper_2005_09824_amd import binding, chain
from tests import layers_oracle as oracle

pytestmark = pytest.mark.gpu

DTYPES = ["float32", "bfloat16", "float16"]


def _torch():
    import torch
    return torch


def _logits(rng, shape, dtype, sigma=2.5):
    torch = _torch()
    x = torch.from_numpy(rng.normal(0, sigma, shape).astype(np.float32)).to(getattr(torch, dtype)).cuda()
    return x, x.double().cpu().numpy()


def check(x64, t, lengths, scale, uniforms, d64, draft_scale, r):
    B, rows, _V = x64.shape
    got = [v.cpu().numpy() for v in r]
    for b in range(B):
        n = rows - 1 if lengths is None else int(lengths[b])
        u = None if uniforms is None else uniforms[b]
        a, token, status = oracle.verify(x64[b], t[b], n, scale, u, None if d64 is None else d64[b], draft_scale)
        want = list(t[b, :a]) + [token] + [-1] * (rows - 1 - a)
        assert (got[0][b], got[2][b], got[1][b].tolist()) == (a, status, want), (b, n, a, token, status, got[0][b], got[1][b])


def _case(rng, B, K, V, dtype, drafted="draft"):
    """Logits of a target and of a draft that nearly knows, tokens drawn from the draft."""
    torch = _torch()
    x, x64 = _logits(rng, (B, K + 1, V), dtype)
    d = torch.from_numpy((0.8 * x64[:, :K] + rng.normal(0, 0.8, (B, K, V))).astype(np.float32)).to(x.dtype).cuda()
    d64 = d.double().cpu().numpy()
    t = (d64 + rng.gumbel(size=d64.shape)).argmax(-1) if drafted == "draft" else x64[:, :K].argmax(-1)
    if drafted != "draft":
        t = np.where(rng.random((B, K)) < 0.7, t, rng.integers(0, V, (B, K)))
    return x, x64, d, d64, t.astype(np.int64), rng.random((B, K + 1)).astype(np.float32)


SHAPES = [(1, 1, 1), (1, 0, 1), (3, 2, 2), (7, 5, 3), (40, 3, 84), (9, 8, 1000), (5, 4, 8191), (4, 2, 8192), (3, 3, 8193), (2, 6, 32000),
          (300, 2, 50), (2, 1, 131072), (1, 70, 33), (6, 0, 40000), (1, 3, 600000)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,K,V", SHAPES)
def test_against_the_rule(B, K, V, dtype):
    torch = _torch()
    rng = np.random.default_rng(B + K + V)
    x, x64, d, d64, t, u = _case(rng, B, K, V, dtype)
    tokens, uniforms = torch.from_numpy(t).cuda(), torch.from_numpy(u).cuda()
    lengths = rng.integers(0, K + 1, B)
    for lens, scale, q_scale in ((None, 1.0, 1.0), (lengths, 0.7, 1.25)):
        check(x64, t, lens, scale, u, d64, q_scale,
              binding.lfmmi_verify_tokens(x, tokens, uniforms, d, lens, scale, q_scale))
    x, x64, _d, _d64, t, u = _case(rng, B, K, V, dtype, "lookup")
    tokens, uniforms = torch.from_numpy(t).cuda().to(torch.int32), torch.from_numpy(u).cuda()
    for lens in (None, lengths):
        check(x64, t, lens, 1.0, u, None, 1.0, binding.lfmmi_verify_tokens(x, tokens, uniforms, lengths=lens))
        check(x64, t, lens, 1.0, None, None, 1.0, binding.lfmmi_verify_tokens(x, tokens, lengths=lens))


@pytest.mark.parametrize("dtype", DTYPES)
def test_ties_go_to_the_lowest_index(dtype):
    torch = _torch()
    V = 20000
    x = torch.zeros((3, 2, V), dtype=getattr(torch, dtype), device="cuda")
    x[0, 0, [7, 9000, 19999]] = 1.0
    x[0, 1, [19999, 8192]] = 1.0
    x[1, 0] = -0.0
    x[1, 0, 5:] = 0.0
    r = binding.lfmmi_verify_tokens(x, torch.tensor([[7], [0], [1]], device="cuda"))
    assert r.tokens.tolist() == [[7, 8192], [0, 0], [0, -1]] and r.accepted.tolist() == [1, 1, 0]


@pytest.mark.parametrize("V", [2, 9000, 40000])
def test_random_numbers_next_to_the_border(V):
    # u as near as float32 comes to p / q from either side: 64 bits decide
    torch = _torch()
    rng = np.random.default_rng(V)
    B = 60
    x, x64, d, d64, t, u = _case(rng, B, 1, V, "float32")
    for b in range(B):
        p, q = oracle.softmax(x64[b, 0], 1.0)[0], oracle.softmax(d64[b, 0], 1.0)[0]
        t[b, 0] = rng.choice(np.flatnonzero(p <= max(0.9, (p / q).min()) * q))
        ratio = np.float32(p[t[b, 0]] / q[t[b, 0]])
        u[b, 0] = [ratio, np.nextafter(ratio, np.float32(0)), np.nextafter(ratio, np.float32(1))][b % 3]
    r = binding.lfmmi_verify_tokens(x, torch.from_numpy(t).cuda(), torch.from_numpy(u).cuda(), d)
    assert 0 < int(r.accepted.sum()) < B
    check(x64, t, None, 1.0, u, d64, 1.0, r)


def test_equal_probabilities():
    # p is 1/2 to the bit and q 1: taken below 1/2, not at it. Two tokens of 1/2 each: drawn by halves
    torch = _torch()
    x = torch.zeros((4, 2, 2), device="cuda")
    d = torch.tensor([0.0, -np.inf], device="cuda").expand(4, 1, 2)
    u = torch.tensor([[0.5, 0.1], [np.nextafter(np.float32(0.5), np.float32(0)), 0.0], [0.0, 0.5], [0.0, 0.49999997]], device="cuda")
    t = torch.zeros((4, 1), dtype=torch.int64, device="cuda")
    for draft in (d, None):
        r = binding.lfmmi_verify_tokens(x, t, u, draft)
        assert r.accepted.tolist() == [0, 1, 1, 1] and r.tokens.tolist() == [[1, -1], [0, 0], [0, 1], [0, 0]]
    # the draft is the target: whatever u below 1 is, everything is taken
    d = torch.randn((4, 1, 50), device="cuda")
    u = torch.full((4, 2), float(np.nextafter(np.float32(1), np.float32(0))), device="cuda")
    r = binding.lfmmi_verify_tokens(torch.cat([d, d], 1), t, u, d)
    assert r.accepted.tolist() == [1] * 4
    # and of a number that is no probability (1 or more) the rule is kept: p - q leaves nothing, p is drawn from
    r = binding.lfmmi_verify_tokens(torch.cat([d, d], 1), t, u + 1, d)
    assert r.accepted.tolist() == [0] * 4 and r.tokens[:, 0].tolist() == [49] * 4 and not r.status.any()


def test_what_rounding_leaves_of_equal_probabilities():
    # p and q are the same but for rounding, and the drafted token is masked out of both: whatever is left of
    # p - q, and whatever the random number is, the token drawn is one that p gives something to
    torch = _torch()
    rng = np.random.default_rng(8)
    B, V = 20000, 8
    x = np.round(rng.normal(0, 4, (B, 2, V)) * 64).astype(np.float32) / 64   # (three times that is exact)
    x[rng.random((B, 2, V)) < 0.2] = -np.inf
    x[:, :, 1] = 0.25
    x[:, :, 0] = -np.inf
    logits = torch.from_numpy(x).cuda()
    u = torch.from_numpy(rng.choice([0.0, 0.3, 0.9, 1.0 - 2.0 ** -24, 1.0], (B, 2)).astype(np.float32)).cuda()
    t = torch.zeros((B, 1), dtype=torch.int64, device="cuda")
    r = binding.lfmmi_verify_tokens(logits, t, u, logits[:, :1] * 3, scale=0.75, draft_scale=0.25)
    assert not r.status.any() and not r.accepted.any() and bool((r.tokens[:, 1] == -1).all())
    assert int(r.tokens[:, 0].min()) > 0
    assert bool(torch.isfinite(logits[:, 0].gather(1, r.tokens[:, :1].long())).all())


@pytest.mark.parametrize("dtype", ["float32", "float16"])
@pytest.mark.parametrize("V", [2100, 4096, 150000])
def test_a_part_that_rounding_alone_leaves(V, dtype):
    # two tokens, the second alone in a part of the row's (a wave takes 2,048 logits); the draft also gives 1e-16
    # and more to a drafted token that the target masks. Every sequence draws a token that the target knows
    torch = _torch()
    rng = np.random.default_rng(V)
    B, far = 400 if V > 10000 else 4000, V - 7
    x = torch.full((B, 2, V), -np.inf, dtype=getattr(torch, dtype), device="cuda")
    x[:, :, 0] = 0.0
    x[:, 0, far] = torch.from_numpy(rng.uniform(-3, 0, B).astype(np.float32)).cuda().to(x.dtype)
    x[0, 0, far] = -0.916799545
    d = x[:, :1].clone()
    d[:, 0, 5] = torch.from_numpy(rng.uniform(-37, -33, B).astype(np.float32)).cuda().to(x.dtype)
    d[0, 0, 5] = -35.7673492
    t = torch.full((B, 1), 5, dtype=torch.int64, device="cuda")
    for last in (0.0, 0.5, 0.9, 1.0):
        u = torch.tensor([0.5, last], device="cuda").expand(B, 2).contiguous()
        r = binding.lfmmi_verify_tokens(x, t, u, d)
        assert not r.status.any() and not r.accepted.any()
        assert bool(((r.tokens[:, 0] == 0) | (r.tokens[:, 0] == far)).all())


def test_tokens_that_cannot_be_drawn():
    torch = _torch()
    V = 10000
    x = torch.full((3, 2, V), -np.inf, device="cuda")
    x[:, :, 9500] = 0.0
    x[:, :, 77] = 0.0
    u = torch.tensor([[0.0, 0.0], [0.0, 0.999], [0.9, 0.0]], device="cuda")
    t = torch.tensor([[5], [77], [9500]], device="cuda")   # p is 0 at 5: never taken, not even with u 0
    r = binding.lfmmi_verify_tokens(x, t, u)
    assert r.accepted.tolist() == [0, 1, 0] and r.tokens.tolist() == [[77, -1], [77, 9500], [77, -1]]
    # a token that the draft gives nothing to is taken if the target gives it anything
    d = torch.full((3, 1, V), -np.inf, device="cuda")
    d[:, :, 3] = 0.0
    r = binding.lfmmi_verify_tokens(x, t, u, d)
    assert r.accepted.tolist() == [0, 1, 1]


def test_flags():
    torch = _torch()
    V, K = 9000, 2
    base = torch.randn((8, K + 1, V), device="cuda")
    x, d = base.clone(), base[:, :K].clone()
    t = d.argmax(-1)
    u = torch.full((8, K + 1), 1e-6, device="cuda")
    x[0, 1] = -np.inf                       # the second row of nothing
    x[1, 0, 8500] = float("nan")
    x[2, 2, 17] = np.inf                    # the row behind the last token
    t[3, 1] = V
    t[4, 0] = -1
    d[5, 1] = -np.inf
    x[6, 2] = float("nan")                  # behind what is looked at
    lengths = [2, 2, 2, 2, 2, 2, 1, 2]
    r = binding.lfmmi_verify_tokens(x, t, u, d, lengths)
    check(x.double().cpu().numpy(), t.cpu().numpy(), lengths, 1.0, u.cpu().numpy(), d.double().cpu().numpy(), 1.0, r)
    assert r.status.tolist() == [1, 2, 2, 4, 4, 1, 0, 0] and r.accepted.tolist() == [1, 0, 2, 1, 0, 1, 1, 2]
    assert (r.tokens[:6].gather(1, r.accepted[:6, None].long()) == -1).all() and int(r.tokens[6, 1]) >= 0
    d[7, 0, 4] = float("nan")
    d[5, 0, 4] = np.inf
    r = binding.lfmmi_verify_tokens(x, t, u, d, lengths)
    assert r.status.tolist() == [1, 2, 2, 4, 4, 2, 0, 2] and r.accepted[7] == 0
    r = binding.lfmmi_verify_tokens(x, t, lengths=lengths)
    check(x.double().cpu().numpy(), t.cpu().numpy(), lengths, 1.0, None, None, 1.0, r)
    assert r.status.tolist() == [1, 2, 2, 4, 4, 0, 0, 0]
    # the type's lowest value is a value: a row of nothing else is a uniform one
    low = torch.full((1, 1, 4), torch.finfo(torch.float32).min, device="cuda")
    r = binding.lfmmi_verify_tokens(low, None, torch.tensor([[0.6]], device="cuda"))
    assert r.tokens.tolist() == [[2]] and r.status.tolist() == [0]


@pytest.mark.parametrize("dtype", DTYPES)
def test_values_that_are_none(dtype):
    # NaN of either sign and +inf, at the beginning, in the middle and at the very end of a row, and in one of -inf
    torch = _torch()
    V = 5000
    base = torch.randn((9, 2, V), device="cuda").to(getattr(torch, dtype))
    minus = (torch.tensor(-4194304, dtype=torch.int32) if dtype == "float32" else torch.tensor(-64, dtype=torch.int16)).view(base.dtype).cuda()
    assert torch.isnan(minus) and torch.signbit(minus)
    for row in (0, 1):
        x = base.clone()
        for b, (at, value) in enumerate(((0, float("nan")), (2500, minus), (V - 1, minus), (0, float("inf")), (V - 1, float("inf")),
                                         (4999, float("nan")), (17, minus))):
            if b == 6:
                x[b, row] = -np.inf
            x[b, row, at] = value
            assert torch.isnan(x[b, row, at]) == np.isnan(float(value))
        x[7, row] = -np.inf
        t = torch.zeros((9, 1), dtype=torch.int64, device="cuda")
        t[:, 0] = x[:, 0].float().nan_to_num(0).argmax(-1)
        u = torch.full((9, 2), 1e-30, device="cuda")
        d = base[:, :1].clone()
        for draft, uniforms in ((d, u), (None, u), (None, None)):
            r = binding.lfmmi_verify_tokens(x, t, uniforms, draft)
            check(x.double().cpu().numpy(), t.cpu().numpy(), None, 1.0, None if uniforms is None else u.cpu().numpy(),
                  None if draft is None else d.double().cpu().numpy(), 1.0, r)
            assert r.status[8] == 0 and (row == 1 or r.status[:8].tolist() == [2] * 7 + [1])
        if row == 0:   # the same in the draft's row
            r = binding.lfmmi_verify_tokens(base, t, u, x[:, :1].contiguous())
            assert r.status.tolist() == [2] * 7 + [1, 0] and not r.accepted[:8].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [1e-6, 0.37, 1e6])
def test_large_and_small_logits(scale, dtype):
    # rows whose largest logit is far from 0, where the next smaller value of the type is far below it
    torch = _torch()
    rng = np.random.default_rng(int(scale * 100) + 1)
    top = 3e4 if dtype == "float16" else 1e30
    x = torch.from_numpy(rng.normal(0, 1, (6, 3, 3000)).astype(np.float32)).to(getattr(torch, dtype)).cuda()
    x[0] += top
    x[1] -= top
    x[2] *= 1e-6
    x[3, :, 2047:] = top
    x[4] *= 1e4
    x[5, :, 1:] = torch.finfo(x.dtype).min
    x[5, :, 0] = -np.inf
    u = rng.random((6, 3)).astype(np.float32)
    t = rng.integers(0, 3000, (6, 2))
    t[:3, 0] = x[:3, 0].double().cpu().numpy().argmax(-1)
    x64 = x.double().cpu().numpy()
    check(x64, t, None, scale, u, x64[:, 1:], scale,
          binding.lfmmi_verify_tokens(x, torch.from_numpy(t).cuda(), torch.from_numpy(u).cuda(), x[:, 1:], scale=scale, draft_scale=scale))
    check(x64, t, None, scale, u, None, 1.0,
          binding.lfmmi_verify_tokens(x, torch.from_numpy(t).cuda(), torch.from_numpy(u).cuda(), scale=scale))


@pytest.mark.parametrize("dtype", DTYPES)
def test_views(dtype):
    torch = _torch()
    rng = np.random.default_rng(5)
    B, K, V = 4, 3, 333
    x, x64, d, d64, t, u = _case(rng, B, K, V, dtype)
    nan = lambda *shape: torch.full(shape, float("nan"), dtype=x.dtype, device="cuda")
    xv, dv = nan(K + 3, B, V + 5)[1:K + 2, :, 3:V + 3].transpose(0, 1), nan(B, K + 1, V + 1)[:, :K, 1:]
    xv.copy_(x)
    dv.copy_(d)
    tokens, uniforms = torch.from_numpy(t).cuda(), torch.from_numpy(u).cuda()
    check(x64, t, None, 1.0, u, d64, 1.0, binding.lfmmi_verify_tokens(xv, tokens, uniforms, dv))
    one, one_d = x[:1, :1].expand(B, K + 1, V), d[:1, :1].expand(B, K, V)
    check(np.broadcast_to(x64[:1, :1], x64.shape), t, None, 1.0, u, np.broadcast_to(d64[:1, :1], d64.shape), 1.0,
          binding.lfmmi_verify_tokens(one, tokens, uniforms, one_d))


def test_what_comes_out_is_distributed_as_the_target():
    # 40,000 sequences of the same rows: shares within 5.5 deviations (8 shares, 3 tests)
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(4)
    B, V = 40000, 8
    row, draft = torch.randn((2, V), generator=gen, device="cuda").mul_(1.5)[:, None]
    p = row.double().softmax(-1)[0]
    for with_draft in (True, False):
        q = draft.double().softmax(-1) if with_draft else torch.full((1, V), 1.0 / V, device="cuda", dtype=torch.float64)
        t = torch.multinomial(q.expand(B, V), 1, generator=gen)
        u = torch.rand((B, 2), generator=gen, device="cuda")
        r = binding.lfmmi_verify_tokens(row.expand(B, 2, V), t, u, draft.expand(B, 1, V) if with_draft else None)
        share = torch.bincount(r.tokens[:, 0].long(), minlength=V).double() / B
        assert bool(((share - p).abs() < 5.5 * (p * (1 - p) / B).sqrt()).all()), (share, p)
    r = binding.lfmmi_verify_tokens(row.expand(B, 1, V), None, torch.rand((B, 1), generator=gen, device="cuda"))
    share = torch.bincount(r.tokens[:, 0].long(), minlength=V).double() / B
    assert bool(((share - p).abs() < 5.5 * (p * (1 - p) / B).sqrt()).all())


def test_outputs_refusals_and_no_sequences():
    torch = _torch()
    x, t = torch.randn((3, 2, 40), device="cuda"), torch.zeros((3, 1), dtype=torch.int64, device="cuda")
    u = torch.rand((3, 2), device="cuda")
    want = binding.lfmmi_verify_tokens(x, t, u)
    out = binding.VerifiedTokens(*(torch.full_like(v, 99) for v in want))
    versions = [v._version for v in out]
    assert binding.lfmmi_verify_tokens(x, t, u, out=out) is out
    assert all(torch.equal(a, b) for a, b in zip(out, want)) and all(v._version > k for v, k in zip(out, versions))
    for args, kw in (((x, None, u), {}), ((x, t[:2], u), {}), ((x, t, u[:, :1]), {}), ((x, t, u.double()), {}), ((x, t, None, x[:, :1]), {}),
                     ((x, t, u, x), {}), ((x, t.float(), u), {}), ((x[0], t, u), {}), ((x, t, u), dict(lengths=[1, 1])),
                     ((x, t, u), dict(out=out._replace(tokens=out.accepted))), ((x[:, :0], None, None), {}),
                     ((x[:, :, ::2], t, u), {}), ((x, t, u, x[:, :1].half()), {})):
        with pytest.raises(ValueError):
            binding.lfmmi_verify_tokens(*args, **kw)
    for kw in (dict(lengths=[1, 2, 0]), dict(scale=0.0), dict(out=out._replace(status=out.accepted))):
        with pytest.raises(binding.LfmmiError):
            binding.lfmmi_verify_tokens(x, t, u, **kw)
    r = binding.lfmmi_verify_tokens(x[:0], t[:0], u[:0])
    assert r.tokens.shape == (0, 2)


def test_captured_and_replayed():
    torch = _torch()
    rng = np.random.default_rng(6)
    x, _x64, d, _d64, t, u = _case(rng, 5, 4, 20000, "bfloat16")
    tokens, uniforms = torch.from_numpy(t).cuda(), torch.from_numpy(u).cuda()
    lengths = [4, 0, 1, 2, 3]
    out = binding.lfmmi_verify_tokens(x, tokens, uniforms, d, lengths)
    greedy = binding.lfmmi_verify_tokens(x, tokens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.lfmmi_verify_tokens(x, tokens, uniforms, d, lengths, out=out)
        binding.lfmmi_verify_tokens(x, tokens, out=greedy)
    for _ in range(4):
        uniforms.copy_(torch.rand((5, 5)))
        x.copy_(x.roll(1, 0))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, binding.lfmmi_verify_tokens(x, tokens, uniforms, d, lengths)))
        assert all(torch.equal(a, b) for a, b in zip(greedy, binding.lfmmi_verify_tokens(x, tokens)))


def test_two_calls_at_once():
    torch = _torch()
    rng = np.random.default_rng(7)
    cases = [_case(rng, 6, 3, 30000, "float16") for _ in range(2)]
    args = [(x, torch.from_numpy(t).cuda(), torch.from_numpy(u).cuda(), d) for x, _a, d, _b, t, u in cases]
    want = [binding.lfmmi_verify_tokens(*a) for a in args]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [binding.lfmmi_verify_tokens(*a, stream=s.cuda_stream) for _ in range(5) for a, s in zip(args, streams)]
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(r, want[i % 2]))


def test_a_long_vocabulary():
    # offsets pass 32 bits: the rows of 2^28 logits of the second sequence begin behind 2^32 bytes
    torch = _torch()
    V = 1 << 28
    x = torch.full((2, 4, V), -np.inf, dtype=torch.float16, device="cuda")
    x[..., V - 1] = 1.0
    x[..., 3] = 1.0
    t = torch.tensor([[3, V - 1, 3]] * 2, device="cuda")
    u = torch.tensor([[0.4, 0.4, 0.6, 0.0], [0.4, 0.4, 0.4, 0.9]], device="cuda")
    r = binding.lfmmi_verify_tokens(x, t, u)
    assert r.accepted.tolist() == [2, 3] and r.tokens.tolist() == [[3, V - 1, V - 1, -1], [3, V - 1, 3, V - 1]]


# ---- the operators together, as they are used

def test_a_training_step():
    # a small model of tokens: embeddings, two blocks with dropout, output layer with the table's own
    # weights, log probabilities, clipping. Against the same in fp64, where every rounding of the fp32 step
    # is worth some 2^-24 of sums of at most a few hundred terms: 1e-4 of the largest gradient
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(1)
    V, D, B, T = 60, 48, 4, 30
    lengths, p = [30, 17, 1, 0], 0.2
    leaves = [torch.randn((V, D), generator=gen, device="cuda").mul_(0.3)]
    leaves += [torch.randn((D, D), generator=gen, device="cuda").mul_(0.15) for _ in range(2)]
    leaves += [torch.ones(D, device="cuda") + 0.1 * torch.randn(D, generator=gen, device="cuda") for _ in range(2)]
    tokens = torch.randint(0, V, (B, T), generator=gen, device="cuda")
    targets = tokens.roll(-1, 1).contiguous()
    targets[:, ::7] = -1

    def step(table, w1, w2, n1, n2):
        h, _status = chain.embed_tokens(table, tokens, lengths, 4.0)
        y, h = chain.add_rms_norm(chain.dropout(h, p, 5, 0), None, n1, 1e-5, lengths)
        y, h = chain.add_rms_norm(torch.tanh(y @ w1), h, n2, 1e-5, lengths, p, 5, 1)
        logits = torch.tanh(y @ w2) @ table.t() * 2
        logp, entropy, _status = chain.token_logprobs(logits, targets, lengths)
        return -(logp.sum() + 0.1 * entropy.sum()) / sum(lengths)

    live = (torch.arange(T)[None] < torch.tensor(lengths)[:, None]).cuda()[..., None]
    masks = [torch.from_numpy(oracle.kept(np.arange(B * T), D, p, 5, k).reshape(B, T, D)).cuda() for k in (0, 1)]
    drop = lambda v, k: v * masks[k] * oracle.factor(p)

    def step64(table, w1, w2, n1, n2):
        norm = lambda v, w: v / (v.square().mean(-1, keepdim=True) + float(np.float32(1e-5))).sqrt() * w * live
        h = drop(table[tokens] * 4.0 * live, 0)
        y = norm(h, n1)
        h = (h + drop(torch.tanh(y @ w1), 1)) * live
        logits = torch.tanh(norm(h, n2) @ w2) @ table.t() * 2
        lp = logits.log_softmax(-1)
        scored = live[..., 0] & (targets >= 0)
        logp = lp.gather(-1, targets.clamp(min=0)[..., None])[..., 0][scored]
        return -(logp.sum() - 0.1 * (lp.exp() * lp).sum(-1)[scored].sum()) / sum(lengths)

    ours = [v.clone().requires_grad_() for v in leaves]
    theirs = [v.cpu().double().requires_grad_() for v in leaves]
    loss = step(*ours)
    loss.backward()
    live, tokens, targets, masks = live.cpu(), tokens.cpu(), targets.cpu(), [m.cpu() for m in masks]
    want = step64(*theirs)
    want.backward()
    assert abs(float(loss.detach()) - float(want.detach())) < 1e-5 * abs(float(want.detach()))
    for a, b in zip(ours, theirs):
        assert float((a.grad.cpu() - b.grad).abs().max()) < 1e-4 * float(b.grad.abs().max())
    total = float(sum(b.grad.square().sum() for b in theirs) ** 0.5)
    assert abs(float(chain.clip_grad_norm(ours, 0.1)) - total) < 1e-4 * total


def test_a_captured_training_step():
    # forward and backward through autograd in one graph, a step on the device that moves the masks; every replay against
    # the eager step of the same number. The warm-up's graphs are gone before the capture begins
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(3)
    V, D, B, T = 90, 72, 3, 20
    lengths = [20, 0, 11]
    leaves = [torch.randn((V, D), generator=gen, device="cuda").mul_(0.3).requires_grad_(),
              torch.ones(D, device="cuda").requires_grad_()]
    tokens = torch.randint(-1, V, (B, T), generator=gen, device="cuda")
    targets = torch.randint(0, V, (B, T), generator=gen, device="cuda")
    grad = torch.randn((B, T), generator=gen, device="cuda")
    number = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step(at):
        table, weight = leaves
        h, _status = chain.embed_tokens(table, tokens, lengths, 2.0)
        y, h = chain.add_rms_norm(chain.dropout(h, 0.2, 5, 1 << 40, at), h, weight, 1e-5, lengths, 0.3, 5, 0, at)
        logp, _entropy, _status = chain.token_logprobs((y + h) @ table.t(), targets, lengths)
        return [logp.detach()] + list(torch.autograd.grad(logp, leaves, grad))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step(number)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(number)
    seen = []
    for k in (0, 3, 1 << 33, 3, -1):
        number.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        want = step(torch.full((1,), k, dtype=torch.int64, device="cuda"))
        for a, b in zip(out, want):
            assert float((a - b).abs().max()) <= 1e-5 * float(b.abs().max())   # (products may be cut otherwise: 90 terms, 2^-24 each, twice)
        seen.append(out[0].clone())
    assert torch.equal(seen[1], seen[3]) and not torch.equal(seen[0], seen[1]) and not torch.equal(seen[2], seen[4])


def test_gradients_of_two_streams_at_once():
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(4)
    B, T, D, V = 8, 400, 512, 700
    made = []
    for k in range(2):
        made.append({"g": torch.randn((B, T, D), generator=gen, device="cuda"),
                     "x": torch.randn((B, T, D), generator=gen, device="cuda"),
                     "tokens": torch.randint(0, V, (B, T), generator=gen, device="cuda")})
    weight = torch.ones(D, device="cuda")

    def call(m, seed):
        r = binding.lfmmi_add_rms_norm(m["x"], m["g"], weight, p=0.1, seed=seed)
        d = binding.lfmmi_add_rms_norm_backward(r.sum, r.rstd, weight, m["g"], m["x"], p=0.1, seed=seed)
        return list(d) + [binding.lfmmi_embed_tokens_backward(d.x, m["tokens"], V)]

    want = [call(m, k) for k, m in enumerate(made)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    got = [[], []]
    for _ in range(5):
        for k, (m, s) in enumerate(zip(made, streams)):
            with torch.cuda.stream(s):
                got[k].append(call(m, k))
    torch.cuda.synchronize()
    for k in range(2):
        for tensors in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(tensors, want[k]))


def test_a_serving_step():
    # embeddings of what was drafted, a norm into 8 bits, a layer, verification, scores of what was taken
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(2)
    V, D, B, K = 500, 128, 6, 3
    table = torch.randn((V, D), generator=gen, device="cuda").bfloat16()
    weight = torch.ones(D, device="cuda")
    layer = torch.randn((D, V), generator=gen, device="cuda") * 0.3
    tokens = torch.randint(0, V, (B, K + 1), generator=gen, device="cuda")
    rows, _status = binding.lfmmi_embed_tokens(table, tokens)
    r = binding.lfmmi_add_rms_norm(rows, rows, weight, quantized=True)
    logits = (r.q.float() * r.q_scale[..., None]) @ layer
    v = binding.lfmmi_verify_tokens(logits, tokens[:, 1:].contiguous(), torch.rand((B, K + 1), generator=gen, device="cuda"))
    check(logits.double().cpu().numpy(), tokens[:, 1:].cpu().numpy(), None, 1.0, None, None, 1.0, binding.lfmmi_verify_tokens(
        logits, tokens[:, 1:].contiguous()))
    scored = binding.lfmmi_token_logprobs(logits, v.tokens, top_k=1)
    assert bool(((v.tokens >= 0) == (scored.logp < 0)).all())
    assert (v.tokens >= 0).sum(1).tolist() == (v.accepted + 1).tolist()
