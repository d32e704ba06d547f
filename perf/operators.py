"""The operators on token log probabilities and on gradients, as they are measured.

A case is a plain dict. Two families:

`"entry": "score"` and `"train"`: log probabilities of given tokens, with entropy and top
alternatives, of logits [batch, frames, vocab] (or [batch, vocab] where `frames` is 0).
`t_lo` / `t_hi`: the range of the sequences' lengths (t_hi == frames; 0: no lengths are
given). `ignored`: the share of rows whose target is -1. `masked`: the share of a row's
vocabulary that a mask takes out (-inf); with `empty` a few rows have everything masked.
`pad`: the columns and rows that the logits are a view without. "score" returns log
probabilities, entropies and the best `top` tokens (no log probabilities of targets where
`targets` is false); "train" returns log probabilities, entropies and the gradient with
respect to the logits for given gradients of both.

`"entry": "norm"` and `"clip"`: the global norm of `tensors` gradients of `elements` values
together, and those gradients scaled so that it is at most 1. `active`: whether it is above
1 before. "clip" writes into buffers of its own, or in place (`in_place`, with a norm below
1: the gradients stay as they are, so that a pass can be repeated).
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
_SIZES = {"float32": 4, "bfloat16": 2, "float16": 2, "mixed": 8.0 / 3.0}


def _rows(**kw):
    case = {"entry": "score", "batch": 1, "frames": 0, "t_lo": 0, "t_hi": 0, "vocab": 32000,
            "dtype": "bfloat16", "top": 0, "targets": True, "ignored": 0.0, "masked": 0.0,
            "empty": False, "pad": 0, "scale": 1.0}
    case.update(kw)
    return case


def _grads(**kw):
    case = {"entry": "clip", "tensors": 40, "elements": 6300000, "dtype": "float32",
            "active": True, "in_place": False}
    case.update(kw)
    return case


def listed():
    return [
        # one step of a decoder that serves a single user: the best alternatives of the
        # next token, before one is chosen. Nothing but latency
        _rows(name="next_token", vocab=32000, top=8, targets=False),
        # a step of a serving batch: what was chosen, its log probability, alternatives
        _rows(name="next_tokens_48", batch=48, vocab=128000, dtype="float16", top=20, scale=1.25),
        # scoring under a grammar: most of an odd vocabulary is masked, some rows wholly
        _rows(name="masked_odd", batch=257, vocab=50021, dtype="float32", top=64, masked=0.6,
              empty=True),
        # scoring prompts of different lengths: a batch of them over a large vocabulary
        _rows(name="score_prompts", batch=8, frames=512, t_lo=100, t_hi=512, vocab=131072, top=5),
        # cross-entropy of a frame alignment beside the sequence loss: the benchmark's
        # default batch, 84 pdfs
        _rows(name="frames_mono", entry="train", batch=64, frames=500, t_lo=100, t_hi=500,
              vocab=84, dtype="float32"),
        # the same over the biphone workload's 3,000 pdfs, in mixed precision
        _rows(name="frames_biphone", entry="train", batch=128, frames=500, t_lo=150, t_hi=500,
              vocab=3000),
        # a training step of a language model or of its policy gradient: prompt tokens are
        # not scored
        _rows(name="train_tokens", entry="train", batch=8192, vocab=65536, ignored=0.25),
        # targets shifted by one and a vocabulary padded for the matrix product: a view
        _rows(name="train_shifted_view", entry="train", batch=6, frames=701, vocab=32003,
              dtype="float16", pad=61, scale=0.7),
        # gradients of an acoustic model of 6.3 million weights, clipped into the buffers
        # that the optimiser reads
        _grads(name="clip_acoustic"),
        # the norm alone, for a log, of gradients of several types
        _grads(name="norm_mixed", entry="norm", tensors=300, elements=300000000, dtype="mixed"),
        # gradients of a large model in mixed precision, norm above the limit
        _grads(name="clip_large", tensors=420, elements=1200000000, dtype="bfloat16"),
        # most steps of a training: the norm is below the limit, nothing has to be written
        _grads(name="clip_quiet", tensors=150, elements=120000000, active=False, in_place=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.35:
        case = _grads(entry=rng.choice(["norm", "clip", "clip"]), tensors=_log_int(rng, 1, 600),
                      dtype=rng.choice(["float32", "bfloat16", "float16", "mixed"]),
                      active=rng.random() < 0.6)
        case["elements"] = max(64 * case["tensors"], _log_int(rng, 1000, 500000000))
        case["in_place"] = case["entry"] == "clip" and not case["active"]
        return case
    case = _rows(entry=rng.choice(["score", "train"]), dtype=rng.choice(list(_DTYPES)),
                 vocab=_log_int(rng, 10, 150000), scale=rng.choice([1.0, 1.0, 0.7, 1.25]))
    rows = _log_int(rng, 1, max(2, min(60000, 260000000 // case["vocab"])))
    if rng.random() < 0.5:
        case["batch"] = _log_int(rng, 1, min(300, rows))
        case["frames"] = max(1, rows // case["batch"])
        if rng.random() < 0.7:
            case["t_lo"], case["t_hi"] = rng.randint(0, case["frames"]), case["frames"]
    else:
        case["batch"] = rows
    if rng.random() < 0.4:
        case["ignored"] = rng.choice([0.05, 0.3, 0.8])
    if rng.random() < 0.3:
        case["masked"], case["empty"] = rng.choice([0.1, 0.5, 0.95]), rng.random() < 0.5
    if rng.random() < 0.3:
        case["pad"] = rng.randint(1, 70)
    if case["entry"] == "score":
        case["top"] = min(rng.choice([0, 1, 5, 20, 64]), case["vocab"])
        case["targets"] = rng.random() < 0.8
        if not case["targets"]:
            case["ignored"] = 0.0
    return case


def _tensor_sizes(case):
    """Sizes of the gradients: two thirds vectors (biases, norms), the rest weights."""
    rng = np.random.default_rng(case["tensors"] * 1000003 + case["elements"])
    n = case["tensors"]
    small = np.where(np.arange(n) % 3 == 0, 0, rng.integers(1, 4097, size=n))
    small = np.minimum(small, max(1, case["elements"] // (4 * n)))
    small[::3] = 0
    share = rng.uniform(0.2, 2.0, size=n) * (small == 0)
    large = np.floor(share / share.sum() * (case["elements"] - small.sum())).astype(np.int64)
    return [int(v) for v in np.maximum(small + large, 1)]


def _prepare_grads(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    rng = np.random.default_rng(seed)
    names = list(_DTYPES) if case["dtype"] == "mixed" else [case["dtype"]]
    sizes = _tensor_sizes(case)
    # layers differ in how large their gradients are; the norm comes to 2.5 or to 0.4
    scales = rng.uniform(0.1, 2.0, size=len(sizes))
    norm = math.sqrt(sum(n * s * s for n, s in zip(sizes, scales)))
    scales *= (2.5 if case["active"] else 0.4) / norm
    grads, flats, outs, out_flats = [None] * len(sizes), [], [None] * len(sizes), []
    for k, name in enumerate(names):  # one bucket of gradients for each type
        mine = list(range(k, len(sizes), len(names)))
        if not mine:
            continue
        flat = torch.randn(sum(sizes[i] for i in mine), generator=gen, device="cuda",
                           dtype=_DTYPES[name])
        flats.append(flat)
        views = flat.split([sizes[i] for i in mine])
        for i, v in zip(mine, views):
            v.mul_(float(scales[i]))
            grads[i] = v
        if case["entry"] == "clip" and not case["in_place"]:
            out_flats.append(torch.empty_like(flat))
            for i, v in zip(mine, out_flats[-1].split([sizes[i] for i in mine])):
                outs[i] = v
    return {"entry": case["entry"], "grads": grads, "flats": flats, "max_norm": 1.0,
            "outs": outs if out_flats else None, "out_flats": out_flats or flats}


def prepare(case, seed):
    if case["entry"] in ("norm", "clip"):
        return _prepare_grads(case, seed)
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    B, T, V = case["batch"], max(1, case["frames"]), case["vocab"]
    dtype = _DTYPES[case["dtype"]]
    base = torch.randn((B, T + (1 if case["pad"] else 0), V + case["pad"]), generator=gen,
                       device="cuda", dtype=dtype)
    base.mul_(2.5)
    x = base[:, :T, :V]
    targets = torch.randint(0, V, (B, T), generator=gen, device="cuda")
    if case["masked"] > 0:
        hidden = torch.rand((1, 1, V), generator=gen, device="cuda") < case["masked"]
        hidden = hidden.expand(B, T, V).scatter(2, targets.unsqueeze(2), False)
        if case["empty"]:
            hidden[::17, ::3] = True
        x.masked_fill_(hidden, -math.inf)
        del hidden
    # a trained model gives the right token a high logit, in some places a very high one
    x.scatter_add_(2, targets.unsqueeze(2),
                   (torch.rand((B, T, 1), generator=gen, device="cuda") * 14.0).to(dtype))
    if case["ignored"] > 0:
        skip = torch.rand((B, T), generator=gen, device="cuda") < case["ignored"]
        targets.masked_fill_(skip, -1)
    lengths = None
    if case["t_hi"] > 0:
        lengths = rng.integers(case["t_lo"], case["t_hi"] + 1, size=B).astype(np.int32)
        lengths[0] = case["t_hi"]
    state = {"entry": case["entry"], "lengths": lengths, "top": case["top"], "scale": case["scale"]}
    if case["entry"] == "train":
        # what the loss hands back: a weight for each token, and one for its entropy
        state["g"] = torch.randn((B, T), generator=gen, device="cuda") / math.sqrt(B * T)
        state["gh"] = torch.rand((B, T), generator=gen, device="cuda") * 0.1 / math.sqrt(B * T)
    if case["frames"] == 0:
        x, targets = x[:, 0], targets[:, 0].contiguous()
        for k in ("g", "gh"):
            if k in state:
                state[k] = state[k][:, 0].contiguous()
    state["x"] = x.detach().requires_grad_() if case["entry"] == "train" else x
    state["targets"] = targets if case["targets"] else None
    return state


def _live(x, targets, lengths):
    """Rows that are scored: inside their sequence, with a target that is not -1."""
    live = torch.ones(x.shape[:-1], dtype=torch.bool, device=x.device)
    if lengths is not None:
        n = torch.as_tensor(lengths, device=x.device).unsqueeze(1)
        live &= torch.arange(x.shape[1], device=x.device).unsqueeze(0) < n
    if targets is not None:
        live &= targets >= 0
    return live


def _top_plain(x, live, top):
    """Ids of the `top` largest values, equal ones by index: the largest of the pairs
    (value, -index), each as one whole number."""
    bits = (x.float() + 0.0).view(torch.int32).to(torch.int64)
    rank = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))
    key = rank * (1 << 32) + ((1 << 31) - torch.arange(x.shape[-1], device=x.device))
    best = key.topk(top, dim=-1).values
    ids = (1 << 31) - (best & 0xFFFFFFFF)
    return torch.where(live.unsqueeze(-1), ids, -1).to(torch.int32)


def _score_plain(state):
    x, targets, scale = state["x"], state["targets"], state["scale"]
    live = _live(x, targets, state["lengths"])
    z = x.float()
    top = z.amax(-1, keepdim=True)
    none = top == -math.inf
    d = (z - top.masked_fill(none, 0.0)) * scale
    e = d.exp()
    s = e.sum(-1, keepdim=True)
    logs = s.log()
    entropy = logs - torch.where(e > 0, e * d, 0.0).sum(-1, keepdim=True) / s
    out = {"entropy": torch.where(live & ~none.squeeze(-1), entropy.squeeze(-1), 0.0),
           "status": (none.squeeze(-1) & live).to(torch.int32)}
    lost = none & live.unsqueeze(-1)
    if targets is not None:
        logp = d.gather(-1, targets.clamp(min=0).unsqueeze(-1)) - logs
        logp = torch.where(lost, -math.inf, logp).squeeze(-1)
        out["logp"] = torch.where(live, logp, 0.0)
    if state["top"]:
        out["top_id"] = _top_plain(x, live, state["top"])
        best = d.gather(-1, out["top_id"].clamp(min=0).to(torch.int64)) - logs
        out["top_logp"] = torch.where(live.unsqueeze(-1), torch.where(lost, -math.inf, best), 0.0)
    return out


def _train_plain(state):
    x, targets, scale = state["x"].detach(), state["targets"], state["scale"]
    live = _live(x, targets, state["lengths"]).unsqueeze(-1)
    z = x.float()
    top = z.amax(-1, keepdim=True)
    none = top == -math.inf
    good = live & ~none
    logp_all = (z - top.masked_fill(none, 0.0)) * scale
    logp_all = logp_all - logp_all.exp().sum(-1, keepdim=True).log()
    p = torch.where(good, logp_all.exp(), 0.0)
    entropy = -torch.where(p > 0, p * logp_all, 0.0).sum(-1, keepdim=True)
    at = targets.clamp(min=0).unsqueeze(-1)
    logp = torch.where(good, logp_all.gather(-1, at), torch.where(live, -math.inf, 0.0))
    g, gh = state["g"].unsqueeze(-1), state["gh"].unsqueeze(-1)
    inner = g + gh * (torch.where(p > 0, logp_all, 0.0) + entropy)
    grad = -p * inner
    grad.scatter_add_(-1, at, torch.where(good, g, 0.0))
    return {"logp": logp.squeeze(-1), "entropy": torch.where(good, entropy, 0.0).squeeze(-1),
            "grad": (grad * scale).to(x.dtype)}


def _norm_plain(grads):
    return torch.stack([g.float().square().sum() for g in grads]).sum().sqrt()


def _clip_plain(state):
    norm = _norm_plain(state["grads"])
    factor = (state["max_norm"] / norm).clamp(max=1.0)
    outs = state["outs"] if state["outs"] is not None else state["grads"]
    [o.copy_(g.float() * factor) for o, g in zip(outs, state["grads"])]
    return {"norm": norm, "grads": state["out_flats"]}


def _run_own(state):
    from paper_2005_09824_amd import binding, chain
    if state["entry"] == "norm":
        return {"norm": binding.lfmmi_grad_norm(state["grads"])}
    if state["entry"] == "clip":
        norm = binding.lfmmi_clip_grads(state["grads"], state["max_norm"], out=state["outs"])
        return {"norm": norm, "grads": state["out_flats"]}
    if state["entry"] == "score":
        r = binding.lfmmi_token_logprobs(state["x"], state["targets"], state["lengths"],
                                         top_k=state["top"], scale=state["scale"])
        out = {"entropy": r.entropy, "status": r.status}
        if r.logp is not None:
            out["logp"] = r.logp
        if state["top"]:
            out["top_id"], out["top_logp"] = r.top_id, r.top_logp
        return out
    logp, entropy, _status = chain.token_logprobs(state["x"], state["targets"], state["lengths"],
                                                  scale=state["scale"])
    (grad,) = torch.autograd.grad((logp, entropy), state["x"], (state["g"], state["gh"]))
    return {"logp": logp.detach(), "entropy": entropy.detach(), "grad": grad}


def run(state):
    if own:
        return _run_own(state)
    if state["entry"] == "norm":
        return {"norm": _norm_plain(state["grads"])}
    if state["entry"] == "clip":
        return _clip_plain(state)
    return _score_plain(state) if state["entry"] == "score" else _train_plain(state)


def work(case):
    """Bytes: each input once, each output once; of logits only the rows that are scored, of
    their gradient every row. Operations: for a logit the difference to the maximum, the
    scale, the exponential, two sums and a product, and as many for its gradient; for a
    gradient a product and a sum, and the product that scales it."""
    size = _SIZES[case["dtype"]]
    if case["entry"] in ("norm", "clip"):
        n = float(sum(_tensor_sizes(case)))
        writes = case["entry"] == "clip" and not case["in_place"]
        return {"bytes": n * size * (2.0 if writes else 1.0) + 4.0,
                "flops": n * (3.0 if writes else 2.0)}
    rows = float(case["batch"] * max(1, case["frames"]))
    live = rows * (1.0 - case["ignored"])
    if case["t_hi"]:
        live *= 0.5 * (case["t_lo"] + case["t_hi"]) / case["t_hi"]
    values = live * case["vocab"]
    small = rows * (12.0 + 8.0 + 8.0 * case["top"])
    if case["entry"] == "train":
        return {"bytes": size * (values + rows * case["vocab"]) + small + 8.0 * rows,
                "flops": 13.0 * values}
    return {"bytes": size * values + small, "flops": 6.0 * values}


def _exact_rows(x, target, live, scale, top, g, gh):
    """The operators' definition in 64 bits, for a few rows."""
    x = x.double()
    n, V = x.shape
    logz = torch.logsumexp(scale * x, dim=1)
    dead = torch.isneginf(logz)
    logz = torch.where(dead, torch.zeros_like(logz), logz)
    l = scale * x - logz.reshape(n, 1)
    p = l.exp()
    plogp = p * l.clamp(min=-1e300)
    entropy = -plogp.sum(dim=1) * live * ~dead
    found = {"entropy": entropy}
    at = torch.arange(n, device=x.device)
    if target is not None:
        logp = l[at, target.clamp(min=0)]
        found["logp"] = logp.masked_fill(dead, -math.inf).masked_fill(~live, 0.0)
    if top:
        best = torch.topk(x, top, dim=1).values * scale - logz.reshape(n, 1)
        found["top_logp"] = best.masked_fill(~live.reshape(n, 1), 0.0)
    if g is not None:
        dlogp = -p
        dlogp[at, target.clamp(min=0)] += 1.0
        dent = -(plogp + p * entropy.reshape(n, 1))
        grad = scale * (g.double().reshape(n, 1) * dlogp + gh.double().reshape(n, 1) * dent)
        found["grad"] = grad.masked_fill(~(live & ~dead).reshape(n, 1), 0.0)
    return found


def exact(case, seed):
    state = prepare(case, seed)
    if case["entry"] in ("norm", "clip"):
        squares = [math.fsum(float(c.double().square().sum()) for c in g.split(1 << 26))
                   for g in state["grads"]]
        norm = math.sqrt(math.fsum(squares))
        found = {"norm": torch.tensor(norm, dtype=torch.float64)}
        if case["entry"] == "clip":
            factor = min(1.0, state["max_norm"] / norm)
            found["grads"] = [f.double() * factor for f in state["flats"]]
        return found
    x = state["x"].detach()
    shape, V = x.shape[:-1], x.shape[-1]
    T = shape[1] if len(shape) == 2 else 1
    rows = x.shape[0] * T
    lengths = state["lengths"]
    inside = torch.ones((x.shape[0], T), dtype=torch.bool)
    if lengths is not None:
        for b, n in enumerate(lengths):
            inside[b, int(n):] = False
    inside = inside.reshape(-1).cuda()
    target = None if state["targets"] is None else state["targets"].reshape(-1)
    if target is not None:
        inside &= target >= 0
    g = state["g"].reshape(-1) if "g" in state else None
    gh = state["gh"].reshape(-1) if "gh" in state else None
    parts = []
    step = max(1, 40000000 // V)
    for a in range(0, rows, step):
        r = torch.arange(a, min(rows, a + step), device=x.device)
        some = x[r // T, r % T] if len(shape) == 2 else x[r]
        pick = lambda v: None if v is None else v[r]
        parts.append(_exact_rows(some, pick(target), inside[r], case["scale"], case["top"],
                                 pick(g), pick(gh)))
    found = {k: torch.cat([q[k] for q in parts]) for k in parts[0]}
    found = {k: v.reshape(shape + v.shape[1:]) for k, v in found.items()}
    if case["entry"] == "score":
        found["status"] = None
        if case["top"]:
            found["top_id"] = None
    return found
