"""The operators around an output layer, as they are measured: token embeddings, dropout, the
residual's addition with a root-mean-square norm, verification of drafted tokens.

A case is a plain dict. `batch`, `frames`: sequences, and rows of each; `t_lo` / `t_hi`: the
range of the sequences' lengths (t_hi == frames; 0: no lengths are given). `width`: values of a
row. Families by `entry`:

`"embed"`, `"embed_train"`: rows of a table [vocab, width] for tokens, times `scale`;
`"embed_train"` returns the table's gradient too, for given gradients of the rows. `spread`: how
tokens fall ("even", or "zipf": the k-th most frequent one 1 / k times as often as the first).
`ignored`: the share of tokens that are -1.

`"dropout"`: rows with a share `p` of their values dropped. `pad`: columns of the tensor that
the rows are a view without.

`"norm"`, `"norm_train"`: residual + dropout(x), its norm, and the gradients with respect to
both and the weight (`"norm_train"`). `residual`: whether there is one. `quantized`: an output
in 8 bits with a scale a row instead of one in the inputs' type.

`"verify"`: `drafts` drafted tokens of each sequence against the target's logits (`t_lo`:
the fewest that a sequence has, `t_hi == drafts`). `draft_logits`: whether the drafting model's
logits are given. `greedy`: no random numbers. `masked`: the share of the vocabulary that a
mask takes out (-inf), with `empty` some rows have everything masked.
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
_SIZES = {"float32": 4, "bfloat16": 2, "float16": 2}
_E4M3_MAX = 448.0
_LEAST_SCALE = 2.0 ** -126
_EPS = 1e-6


def _case(entry, kw, **base):
    case = {"entry": entry, "batch": 1, "frames": 1, "t_lo": 0, "t_hi": 0, "dtype": "bfloat16"}
    case.update(base)
    case.update(kw)
    return case


def _embed(entry="embed", **kw):
    return _case(entry, kw, vocab=32000, width=1024, scale=1.0, spread="zipf", ignored=0.0)


def _dropout(**kw):
    return _case("dropout", kw, width=1024, p=0.1, pad=0)


def _norm(entry="norm", **kw):
    return _case(entry, kw, width=1024, p=0.0, residual=True, quantized=False)


def _verify(**kw):
    return _case("verify", kw, drafts=4, vocab=32000, scale=1.0, draft_logits=True, greedy=False,
                 masked=0.0, empty=False)


def listed():
    return [
        # one step of a serving batch: the rows of the tokens chosen last. Nothing but latency
        _embed(name="embed_step", batch=48, vocab=128000, width=4096),
        # embeddings of an alignment's 84 pdfs beside the acoustic features: few rows, each the sum
        # of hundreds of gradients
        _embed("embed_train", name="embed_pdfs", batch=64, frames=500, t_lo=100, t_hi=500,
               vocab=84, width=640, dtype="float32", spread="even"),
        # a training step of a language model: the gradient of a large table, most of it zeros,
        # some tokens very frequent, prompts padded
        _embed("embed_train", name="embed_tokens", batch=32, frames=1024, t_lo=300, t_hi=1024,
               vocab=65536, width=2048, scale=45.25, ignored=0.05),
        # dropout of an acoustic model's hidden layer
        _dropout(name="dropout_hidden", batch=64, frames=500, width=640, dtype="float32"),
        # dropout of a wide layer's output in mixed precision, a view of an odd width
        _dropout(name="dropout_wide", batch=16, frames=1024, width=8189, pad=3, p=0.2),
        # serving: eight requests' single tokens in front of a layer in 8 bits
        _norm(name="norm_step", batch=8, width=4096, quantized=True),
        # a prompt of odd length and width in front of a layer in 8 bits
        _norm(name="norm_prompt", batch=1, frames=1021, width=5003, dtype="float16", quantized=True),
        # the end of a block of an acoustic model, lengths unequal
        _norm("norm_train", name="norm_frames", batch=64, frames=500, t_lo=100, t_hi=500,
              width=640, dtype="float32", p=0.1),
        # the same of a large model in mixed precision
        _norm("norm_train", name="norm_wide", batch=16, frames=1024, width=8192, p=0.1),
        # a single user's request with four drafted tokens. Nothing but latency
        _verify(name="verify_one", vocab=32000),
        # a serving batch with up to six drafted tokens each
        _verify(name="verify_batch", batch=48, drafts=6, t_lo=0, t_hi=6, vocab=128000,
                dtype="float16", scale=1.25),
        # tokens drafted by looking them up in the prompt (no logits), under a grammar
        _verify(name="verify_lookup", batch=130, drafts=3, vocab=50021, dtype="float32",
                draft_logits=False, masked=0.6, empty=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rows(rng, case, rows):
    """Rows as a batch of sequences, or one token of each."""
    case["batch"] = rows
    if rng.random() < 0.6:
        case["batch"] = _log_int(rng, 1, min(300, rows))
        case["frames"] = max(1, rows // case["batch"])
        if rng.random() < 0.6:
            case["t_lo"], case["t_hi"] = rng.randint(0, case["frames"]), case["frames"]
    return case


def draw(rng):
    entry = rng.choice(["embed", "embed_train", "embed_train", "dropout", "norm", "norm_train",
                        "norm_train", "verify", "verify"])
    dtype = rng.choice(list(_DTYPES))
    if entry == "verify":
        case = _verify(dtype=dtype, batch=_log_int(rng, 1, 200), drafts=rng.choice([0, 1, 2, 3, 4, 5, 8]),
                       scale=rng.choice([1.0, 1.0, 0.7, 1.25]), draft_logits=rng.random() < 0.6,
                       greedy=rng.random() < 0.25)
        case["draft_logits"] = case["draft_logits"] and not case["greedy"]
        rows = case["batch"] * (case["drafts"] + 1)
        case["vocab"] = _log_int(rng, 10, min(150000, max(11, 40000000 // rows)))
        if rng.random() < 0.6:
            case["t_lo"], case["t_hi"] = rng.randint(0, case["drafts"]), case["drafts"]
        if rng.random() < 0.4:
            case["masked"], case["empty"] = rng.choice([0.1, 0.5, 0.95]), rng.random() < 0.4
        return case
    width = _log_int(rng, 16, 16000)
    rows = _log_int(rng, 1, max(2, min(70000, 60000000 // width)))
    if entry == "dropout":
        return _dropout(batch=rows, width=width, dtype=dtype, p=rng.choice([0.02, 0.05, 0.1, 0.3, 0.5]),
                        pad=rng.choice([0, 0, 0, rng.randint(1, 40)]))
    if entry in ("norm", "norm_train"):
        case = _norm(entry, width=width, dtype=dtype, residual=rng.random() < 0.8,
                     p=rng.choice([0.0, 0.1, 0.25]) if entry == "norm_train" else 0.0,
                     quantized=entry == "norm" and rng.random() < 0.5)
        return _draw_rows(rng, case, rows)
    case = _embed(entry, width=width, dtype=dtype, scale=rng.choice([1.0, 32.0, 0.5]),
                  vocab=_log_int(rng, 10, min(200000, max(11, 60000000 // width))),
                  spread=rng.choice(["even", "zipf"]), ignored=rng.choice([0.0, 0.0, 0.1, 0.6]))
    return _draw_rows(rng, case, rows)


def _randn(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _lengths(case, rng, frames):
    if case["t_hi"] == 0:
        return None
    lengths = rng.integers(case["t_lo"], case["t_hi"] + 1, size=case["batch"]).astype(np.int32)
    lengths[0] = case["t_hi"]
    return np.minimum(lengths, frames)


def _prepare_verify(case, rng, gen):
    B, K, V, dtype = case["batch"], case["drafts"], case["vocab"], _DTYPES[case["dtype"]]
    x = _randn(gen, (B, K + 1, V), dtype).mul_(2.5)
    # the target is sure of some tokens
    sure = torch.randint(0, V, (B, K + 1, 1), generator=gen, device="cuda")
    x.scatter_add_(2, sure, (torch.rand((B, K + 1, 1), generator=gen, device="cuda") * 14.0).to(dtype))
    hidden = torch.rand((1, 1, V), generator=gen, device="cuda") < case["masked"]
    hidden[..., V // 2] = False
    x.masked_fill_(hidden, -math.inf)
    state = {"x": x, "draft": None, "uniforms": None, "scale": case["scale"],
             "lengths": _lengths(case, rng, K) if K else None, "entry": "verify"}
    if case["draft_logits"]:
        # a smaller model that nearly knows, and tokens drawn from what it gives
        draft = (x[:, :K].float() * 0.9 + torch.randn((B, K, V), generator=gen, device="cuda") * 0.6)
        state["draft"] = draft.to(dtype).contiguous()
        noise = -torch.log(-torch.log(torch.rand((B, K, V), generator=gen, device="cuda").clamp(1e-20, 1 - 1e-7)))
        drafted = (state["draft"].float() * case["scale"] + noise).argmax(-1)
    else:
        guess = torch.randint(0, V, (B, K), generator=gen, device="cuda")
        right = torch.rand((B, K), generator=gen, device="cuda") < 0.7
        drafted = torch.where(right, x[:, :K].float().argmax(-1), guess)
    state["drafted"] = drafted.contiguous()
    if not case["greedy"]:
        state["uniforms"] = torch.rand((B, K + 1), generator=gen, device="cuda")
    if case["empty"]:
        x[::7, K // 2] = -math.inf
    return state


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    if case["entry"] == "verify":
        return _prepare_verify(case, rng, gen)
    B, T, D, dtype = case["batch"], case["frames"], case["width"], _DTYPES[case["dtype"]]
    state = {"entry": case["entry"], "lengths": _lengths(case, rng, T)}
    if case["entry"] in ("embed", "embed_train"):
        V = case["vocab"]
        state["table"] = _randn(gen, (V, D), dtype)
        u = torch.rand((B, T), generator=gen, device="cuda", dtype=torch.float64)
        rank = (V * u if case["spread"] == "even" else torch.exp(u * math.log(V + 1.0)) - 1.0)
        order = torch.randperm(V, generator=gen, device="cuda")
        tokens = order[rank.to(torch.int64).clamp(0, V - 1)]
        if case["ignored"] > 0:
            tokens.masked_fill_(torch.rand((B, T), generator=gen, device="cuda") < case["ignored"], -1)
        state["tokens"], state["scale"] = tokens.contiguous(), case["scale"]
        if case["entry"] == "embed_train":
            state["grad_out"] = _randn(gen, (B, T, D), dtype)
        return state
    state["p"], state["seed"], state["offset"] = case.get("p", 0.0), int(rng.integers(1 << 62)), int(rng.integers(1 << 40))
    if case["entry"] == "dropout":
        state["x"] = _randn(gen, (B * T, D + case["pad"]), dtype)[:, case["pad"]:]
        return state
    # a residual stream grows through the layers; a few of its channels are large
    state["x"] = _randn(gen, (B, T, D), dtype)
    state["residual"] = None
    if case["residual"]:
        state["residual"] = _randn(gen, (B, T, D), dtype).mul_(3.0)
        state["residual"][..., ::97] *= 8.0
    state["weight"] = 1.0 + 0.2 * _randn(gen, (D,), torch.float32)
    state["quantized"] = case["quantized"]
    if case["entry"] == "norm_train":
        state["grad_y"] = _randn(gen, (B, T, D), dtype)
        state["grad_sum"] = _randn(gen, (B, T, D), dtype) if case["residual"] else None
    return state


# ---- plain forms

def _inside(shape, lengths, device):
    inside = torch.ones(shape[:2], dtype=torch.bool, device=device)
    if lengths is not None:
        n = torch.as_tensor(lengths, device=device).unsqueeze(1)
        inside &= torch.arange(shape[1], device=device).unsqueeze(0) < n
    return inside


def _embed_plain(state):
    table, tokens, scale = state["table"], state["tokens"], state["scale"]
    live = _inside(tokens.shape, state["lengths"], table.device) & (tokens >= 0)
    at = torch.where(live, tokens, 0)
    out = {"out": torch.where(live.unsqueeze(-1), table[at].float() * scale, 0.0).to(table.dtype)}
    if state["entry"] == "embed_train":
        g = torch.where(live.unsqueeze(-1), state["grad_out"].float(), 0.0).reshape(-1, table.shape[1])
        grad = torch.zeros(table.shape, dtype=torch.float32, device=table.device)
        grad.index_add_(0, at.reshape(-1), g)
        out["grad"] = (grad * scale).to(table.dtype)
    return out


def _times(a, m):
    """The high and the low 32 bits of a * m, of whole numbers below 2^32."""
    low = a * (m & 0xFFFF)
    both = a * (m >> 16) + (low >> 16)
    return both >> 16, ((both & 0xFFFF) << 16) | (low & 0xFFFF)


def _philox(c0, c1, c2, c3, seed):
    """Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011) of counters (tensors, or numbers)."""
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        (h0, l0), (h1, l1) = _times(c0, 0xD2511F53), _times(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c0, c1, c2, c3


def _threshold(p):
    return int(np.rint(float(np.float32(p)) * 65536.0))


def _kept(rows, width, state, device):
    """What is kept of [rows, width]: eight values to a block of 128 bits, 16 bits a value."""
    blocks = (width + 7) // 8
    column = torch.arange(blocks, device=device).unsqueeze(0).expand(rows, blocks)
    row = torch.arange(rows, device=device).unsqueeze(1).expand(rows, blocks)
    words = _philox(column, row, state["offset"] & 0xFFFFFFFF, state["offset"] >> 32, state["seed"])
    halves = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], dim=-1)
    return (halves >= _threshold(state["p"])).reshape(rows, blocks * 8)[:, :width]


def _dropped(x, state):
    """x (float32) with what dropout leaves of it."""
    k = _threshold(state["p"])
    if k == 0:
        return x
    kept = _kept(x.numel() // x.shape[-1], x.shape[-1], state, x.device).reshape(x.shape)
    return torch.where(kept, x * float(np.float32(65536.0 / (65536 - k))), 0.0)


def _norm_plain(state):
    x, residual, weight = state["x"], state["residual"], state["weight"]
    live = _inside(x.shape, state["lengths"], x.device).unsqueeze(-1)
    h = _dropped(x.float(), state)
    if residual is not None:
        h = h + residual.float()
    h = torch.where(live, h, 0.0).to(x.dtype)
    out = {} if residual is None and state["p"] == 0 else {"sum": h}
    h = h.float()
    rstd = (h.square().mean(-1, keepdim=True) + _EPS).rsqrt()
    y = torch.where(live, h * rstd * weight, 0.0)
    if state["quantized"]:
        scale = torch.where(live, (y.abs().amax(-1, keepdim=True) / _E4M3_MAX).clamp(min=_LEAST_SCALE), 0.0)
        q = torch.where(live, y / scale, 0.0)
        out["q"] = q.clamp(-_E4M3_MAX, _E4M3_MAX).to(torch.float8_e4m3fn)
        out["q_scale"] = scale.squeeze(-1)
    else:
        out["y"] = y.to(x.dtype)
    if state["entry"] == "norm_train":
        dy = torch.where(live, state["grad_y"].float(), 0.0)
        out["grad_weight"] = (dy * h * rstd).sum((0, 1))
        g = dy * weight
        dh = rstd * (g - h * rstd.square() * (g * h).mean(-1, keepdim=True))
        if state["grad_sum"] is not None:
            dh = dh + torch.where(live, state["grad_sum"].float(), 0.0)
        out["grad_x"] = _dropped(dh, state).to(x.dtype)
        if residual is not None:
            out["grad_residual"] = dh.to(x.dtype)
    return out


def _softmax64(x, scale):
    """Probabilities of rows in 64 bits (0 in a row of nothing but -inf), and those rows."""
    x = x.double()
    top = x.amax(-1, keepdim=True)
    none = top == -math.inf
    e = ((x - top.masked_fill(none, 0.0)) * float(np.float32(scale))).exp()
    return e / e.sum(-1, keepdim=True).masked_fill(none, 1.0), none.squeeze(-1)


def _first_largest(x):
    """The lowest index of the largest value of rows."""
    index = torch.arange(x.shape[-1], device=x.device)
    return torch.where(x == x.amax(-1, keepdim=True), index, x.shape[-1]).amin(-1)


def _verify_plain(state):
    x, drafted, draft = state["x"], state["drafted"], state["draft"]
    B, K, V = x.shape[0], x.shape[1] - 1, x.shape[2]
    n = torch.full((B,), K, device=x.device)
    if state["lengths"] is not None:
        n = torch.as_tensor(state["lengths"], device=x.device).to(torch.int64)
    at = torch.arange(K + 1, device=x.device).unsqueeze(0)
    column = drafted.unsqueeze(-1)
    if state["uniforms"] is None:
        none = x.amax(-1) == -math.inf
        best = _first_largest(x)
        good = drafted == best[:, :K]
    else:
        p, none = _softmax64(x, state["scale"])
        u = state["uniforms"].double()
        here = p[:, :K].gather(-1, column).squeeze(-1)
        if draft is None:
            good = u[:, :K] < here
        else:
            q, none_q = _softmax64(draft, state["scale"])
            good = u[:, :K] * q.gather(-1, column).squeeze(-1) < here
            none[:, :K] |= none_q
    # the first row that is not taken, or the one behind the last drafted token
    ends = torch.ones((B, K + 1), dtype=torch.bool, device=x.device)
    ends[:, :K] = ~good | none[:, :K] | (at[:, :K] >= n.unsqueeze(1))
    accepted = torch.where(ends, at, K + 1).amin(1)
    lost = none.gather(1, accepted.unsqueeze(1)).squeeze(1)
    row = accepted.reshape(B, 1, 1)
    if state["uniforms"] is None:
        token = best.gather(1, accepted.unsqueeze(1)).squeeze(1)
    else:
        weights = p.gather(1, row.expand(B, 1, V)).squeeze(1)
        if K > 0:
            r = row.clamp(max=K - 1)
            if draft is None:
                less = torch.zeros_like(weights).scatter_(1, column.gather(1, r).squeeze(2), 1.0)
            else:
                less = q.gather(1, r.expand(B, 1, V)).squeeze(1)
            rest = torch.where((accepted < n).unsqueeze(1), (weights - less).clamp(min=0.0), weights)
            weights = torch.where(rest.sum(1, keepdim=True) > 0, rest, weights)
        cum = weights.cumsum(1)
        token = (cum <= u[:, K:] * cum[:, -1:]).sum(1).clamp(max=V - 1)
    token = torch.where(lost, -1, token)
    tokens = torch.cat([drafted, drafted.new_full((B, 1), -1)], 1)
    tokens = torch.where(at < accepted.unsqueeze(1), tokens, torch.where(at == accepted.unsqueeze(1), token.unsqueeze(1), -1))
    return {"accepted": accepted.to(torch.int32), "tokens": tokens.to(torch.int32), "status": lost.to(torch.int32)}


def _run_own(state):
    from paper_2005_09824_amd import binding
    entry = state["entry"]
    if entry == "verify":
        r = binding.lfmmi_verify_tokens(state["x"], state["drafted"], state["uniforms"], state["draft"],
                                        lengths=state["lengths"], scale=state["scale"],
                                        draft_scale=state["scale"])
        return {"accepted": r.accepted, "tokens": r.tokens, "status": r.status}
    if entry == "dropout":
        return {"y": binding.lfmmi_dropout(state["x"], state["p"], state["seed"], state["offset"])}
    if entry in ("embed", "embed_train"):
        rows, _status = binding.lfmmi_embed_tokens(state["table"], state["tokens"], state["lengths"],
                                                   scale=state["scale"])
        out = {"out": rows}
        if entry == "embed_train":
            out["grad"] = binding.lfmmi_embed_tokens_backward(
                state["grad_out"], state["tokens"], state["table"].shape[0], state["lengths"],
                scale=state["scale"])
        return out
    random = {"p": state["p"], "seed": state["seed"], "offset": state["offset"]}
    r = binding.lfmmi_add_rms_norm(state["x"], state["residual"], state["weight"], eps=_EPS,
                                   lengths=state["lengths"], quantized=state["quantized"], **random)
    out = {} if state["residual"] is None and state["p"] == 0 else {"sum": r.sum}
    if state["quantized"]:
        out["q"], out["q_scale"] = r.q, r.q_scale
    else:
        out["y"] = r.y
    if entry == "norm_train":
        g = binding.lfmmi_add_rms_norm_backward(r.sum, r.rstd, state["weight"], state["grad_y"],
                                                state["grad_sum"], lengths=state["lengths"],
                                                residual=state["residual"] is not None, **random)
        out["grad_x"], out["grad_weight"] = g.x, g.weight
        if state["residual"] is not None:
            out["grad_residual"] = g.residual
    return out


def run(state):
    if own:
        return _run_own(state)
    if state["entry"] == "verify":
        return _verify_plain(state)
    if state["entry"] == "dropout":
        return {"y": _dropped(state["x"].float(), state).to(state["x"].dtype)}
    return _norm_plain(state) if state["entry"].startswith("norm") else _embed_plain(state)


def work(case):
    """Bytes: each input once, each output once; of rows that lie behind a sequence's end only
    the outputs. Operations: those of the formulas, an exponential as one, and 25 for the
    128 random bits of eight values (a product of 32 bits in ten rounds twice, and what joins them)
    each."""
    size, B, T = _SIZES[case["dtype"]], case["batch"], case["frames"]
    share = 0.5 * (case["t_lo"] + case["t_hi"]) / case["t_hi"] if case["t_hi"] else 1.0
    if case["entry"] == "verify":
        drafts = B * case["drafts"] * share
        rows = drafts + B + (drafts if case["draft_logits"] else 0.0)
        values = rows * case["vocab"]
        return {"bytes": size * values + 16.0 * drafts + 12.0 * B, "flops": 4.0 * values}
    rows, D = float(B * T), case["width"]
    values, live = rows * D, rows * D * share
    bits = 25.0 if case.get("p") else 0.0
    if case["entry"] == "dropout":
        return {"bytes": 2.0 * size * values, "flops": (1.0 + bits) * values}
    if case["entry"] in ("embed", "embed_train"):
        live *= 1.0 - case["ignored"]
        table = float(case["vocab"] * D)
        moved = size * (min(live, table) + values) + 8.0 * rows
        if case["entry"] == "embed":
            return {"bytes": moved, "flops": live}
        return {"bytes": moved + size * (live + table) + 8.0 * rows, "flops": 3.0 * live}
    forward = live * size * (2.0 if case["residual"] else 1.0)
    has_sum = case["residual"] or case["p"] > 0
    forward += values * ((1.0 if case["quantized"] else size) + (size if has_sum else 0.0)) + 4.0 * D
    if case["entry"] == "norm":
        return {"bytes": forward, "flops": (6.0 + bits) * live}
    backward = live * size * (3.0 if case["residual"] else 2.0) + values * size * (2.0 if case["residual"] else 1.0)
    return {"bytes": forward + backward + 8.0 * D, "flops": (18.0 + 2.0 * bits) * live}


# ---- the definitions in 64 bits

def _exact_kept(rows, width, p, seed, offset):
    """The same choice, block by block on the host with products of 64 bits."""
    blocks = (width + 7) // 8
    low = np.uint64(0xFFFFFFFF)
    at = np.arange(rows * blocks, dtype=np.uint64)
    a, b = at % np.uint64(blocks), at // np.uint64(blocks)
    c = np.full_like(at, offset & 0xFFFFFFFF)
    d = np.full_like(at, offset >> 32)
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        first, second = a * np.uint64(0xD2511F53), c * np.uint64(0xCD9E8D57)
        a, b, c, d = ((second >> np.uint64(32)) ^ b ^ np.uint64(key[0]), second & low,
                      (first >> np.uint64(32)) ^ d ^ np.uint64(key[1]), first & low)
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    words = np.stack([a, b, c, d], 1).astype("<u4")
    kept = words.view("<u2").reshape(rows, blocks * 8)[:, :width] >= int(np.rint(float(np.float32(p)) * 65536))
    return torch.from_numpy(kept).cuda()


def _exact_dropped(v, state):
    part = int(np.rint(float(np.float32(state["p"])) * 65536)) / 65536
    if part == 0:
        return v
    flat = v.reshape(-1, v.shape[-1])
    kept = _exact_kept(flat.shape[0], flat.shape[1], state["p"], state["seed"], state["offset"])
    return (flat * kept / (1.0 - part)).reshape(v.shape)


def _exact_norm(case, state):
    x, weight = state["x"], state["weight"].double()
    h = _exact_dropped(x.double(), state)
    if state["residual"] is not None:
        h += state["residual"].double()
    if state["lengths"] is not None:
        for b, n in enumerate(state["lengths"]):
            h[b, int(n):] = 0.0
    found = {} if state["residual"] is None and state["p"] == 0 else {"sum": h}
    v = h.to(x.dtype).double()  # the norm is that of the sum as it is kept
    size = torch.sqrt(torch.sum(v * v, -1, keepdim=True) / v.shape[-1] + _EPS)
    y = v / size * weight
    if state["quantized"]:
        scale = torch.clamp(y.abs().amax(-1) / _E4M3_MAX, min=_LEAST_SCALE)
        found["q"] = y / scale.unsqueeze(-1)
        if state["lengths"] is not None:
            for b, n in enumerate(state["lengths"]):
                scale[b, int(n):] = 0.0
        found["q_scale"] = scale
    else:
        found["y"] = y
    if case["entry"] == "norm_train":
        dy = state["grad_y"].double()
        if state["lengths"] is not None:
            for b, n in enumerate(state["lengths"]):
                dy[b, int(n):] = 0.0
        unit = v / size
        found["grad_weight"] = torch.sum((dy * unit).reshape(-1, v.shape[-1]), 0)
        dy = dy * weight
        dh = (dy - unit * torch.mean(dy * unit, -1, keepdim=True)) / size
        if state["grad_sum"] is not None:
            dsum = state["grad_sum"].double()
            if state["lengths"] is not None:
                for b, n in enumerate(state["lengths"]):
                    dsum[b, int(n):] = 0.0
            dh += dsum
            found["grad_residual"] = dh
        found["grad_x"] = _exact_dropped(dh, state)
    return found


def exact(case, seed):
    if case["entry"] == "verify":
        return None  # whole numbers
    state = prepare(case, seed)
    if case["entry"] == "dropout":
        return {"y": _exact_dropped(state["x"].double(), state)}
    if case["entry"].startswith("norm"):
        return _exact_norm(case, state)
    tokens = state["tokens"].cpu().numpy().copy()
    if state["lengths"] is not None:
        for b, n in enumerate(state["lengths"]):
            tokens[b, int(n):] = -1
    flat = torch.from_numpy(tokens.reshape(-1)).cuda()
    rows = torch.nonzero(flat >= 0).reshape(-1)
    V, D = state["table"].shape
    out = torch.zeros((flat.numel(), D), dtype=torch.float64, device="cuda")
    out[rows] = state["table"].double()[flat[rows]] * case["scale"]
    found = {"out": out.reshape(tokens.shape + (D,))}
    if case["entry"] == "embed_train":
        # every token's rows next to each other, and the difference of their running sums
        order = rows[torch.argsort(flat[rows], stable=True)]
        ends = torch.searchsorted(flat[order], torch.arange(V, device="cuda"), right=True)
        g = state["grad_out"].reshape(-1, D)
        grad = torch.empty((V, D), dtype=torch.float64, device="cuda")
        step = max(1, 100000000 // max(1, order.numel()))
        for a in range(0, D, step):
            sums = torch.nn.functional.pad(g[order, a:a + step].double().cumsum(0), (0, 0, 1, 0))
            grad[:, a:a + step] = torch.diff(sums[ends], dim=0, prepend=sums[:1])
        found["grad"] = grad * case["scale"]
    return found
