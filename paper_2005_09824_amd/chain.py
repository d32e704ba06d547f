"""LF-MMI objective as a torch.autograd.Function on top of the C ABI (Eq. 2, Eq. 3), and
what a training step uses beside it: log probabilities of given tokens, clipping of
gradients to a norm, and in front of the output layer token embeddings, dropout and the end
of a residual block.

All of them may be captured into a HIP graph, backward passes too (torch.autograd.grad, or leaves whose
gradients were never accumulated outside). Before a capture let every eager autograd graph of the same
leaves go: torch ties a leaf's accumulation of gradients to the stream that it first ran on, and a captured
backward pass that meets such a node can end the process.

Argument marshalling only: both forward-backward passes, the objective and its
gradient with respect to the logits all come out of lfmmi_loss; this
file stores that gradient for backward() and scales it by the incoming gradient.
"""
from __future__ import annotations

import numpy as np

from . import binding


def _function_class():
    import torch

    class _ChainObjective(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, lengths, num_graphs, den_graph, leak):
            x = logits.detach()
            if x.dtype != torch.float32 or not x.is_contiguous():
                x = x.float().contiguous()
            # numerator minus denominator (Eq. 2 / Eq. 3), one call
            objf, grad, status = binding.lfmmi_loss(num_graphs, den_graph, x, lengths, leak)
            ctx.save_for_backward(grad)
            ctx.logits_dtype = logits.dtype
            ctx.mark_non_differentiable(status)
            return objf, status

        @staticmethod
        def backward(ctx, grad_objf, _grad_status):
            (grad,) = ctx.saved_tensors
            g = grad * grad_objf.reshape(-1, 1, 1).to(grad.dtype)
            return g.to(ctx.logits_dtype), None, None, None, None

    return _ChainObjective


_cls = None


def chain_objective(logits, lengths, num_graphs, den_graph, leak=1e-5):
    """Per-sequence objective log p(num) - log p(den) of Eq. 2, differentiable in `logits`.

    logits: CUDA float tensor [B, T, P]; lengths: host ints [B]; num_graphs: a batch
    handle with one numerator graph per sequence; den_graph: the shared denominator
    handle. Returns (objf [B], status [B]); the gradient is Eq. 3, the difference
    of the numerator and denominator pdf occupancies."""
    global _cls
    if _cls is None:
        _cls = _function_class()
    return _cls.apply(logits, np.asarray(lengths, dtype=np.int32), num_graphs, den_graph, float(leak))


def _token_class():
    import torch
    from torch.autograd.function import once_differentiable

    class _TokenLogprobs(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, targets, lengths, scale):
            ctx.set_materialize_grads(False)  # what the loss does not use costs nothing
            r = binding.lfmmi_token_logprobs(logits, targets, lengths, scale=scale)
            ctx.save_for_backward(logits, targets, r.stats, r.entropy)
            ctx.lengths, ctx.scale = lengths, scale
            ctx.mark_non_differentiable(r.status)
            return r.logp, r.entropy, r.status

        @staticmethod
        @once_differentiable
        def backward(ctx, grad_logp, grad_entropy, _grad_status):
            if grad_logp is None and grad_entropy is None:
                return None, None, None, None
            logits, targets, stats, entropy = ctx.saved_tensors
            as_rows = lambda g: None if g is None else g.float().contiguous()
            grad = binding.lfmmi_token_logprobs_backward(
                logits, targets, stats, entropy, as_rows(grad_logp), as_rows(grad_entropy),
                ctx.lengths, ctx.scale)
            return grad, None, None, None

    return _TokenLogprobs


_token_cls = None


def token_logprobs(logits, targets, lengths=None, scale=1.0):
    """Log probabilities that rows of logits give to their target tokens (or pdfs, of a frame
    alignment), and the rows' entropies, both differentiable in `logits`.

    logits: CUDA float tensor [B, T, V] or [B, V]; targets: int32 or
    int64 CUDA tensor [B, T] or [B], negative where a row is not scored; lengths: host ints [B]
    or None; scale: what logits are multiplied by. Returns (logp, entropy, status), rows that
    are not scored 0; rows flagged in `status` (nothing but -inf, a NaN or +inf
    logit, a target out of range) have a log probability that is not finite, and gradient 0."""
    global _token_cls
    if targets is None:
        raise ValueError("log probabilities of tokens need targets")
    if _token_cls is None:
        _token_cls = _token_class()
    if lengths is not None:
        lengths = np.array(lengths, dtype=np.int32)  # (a copy: backward reads it)
    if logits.dtype not in binding._dtype_codes():
        logits = logits.float()
    if logits.dim() and logits.shape[-1] > 1 and logits.stride(-1) != 1:
        logits = logits.contiguous()
    return _token_cls.apply(logits, targets.contiguous(), lengths, float(scale))


def _rows_in_order(x):
    """x with the values of a row next to each other, in a type of the library's."""
    if x.dtype not in binding._dtype_codes():
        x = x.float()
    return x.contiguous() if x.dim() and x.shape[-1] > 1 and x.stride(-1) != 1 else x


def _embed_class():
    import torch
    from torch.autograd.function import once_differentiable

    class _EmbedTokens(torch.autograd.Function):
        @staticmethod
        def forward(ctx, table, tokens, lengths, scale):
            rows, status = binding.lfmmi_embed_tokens(table, tokens, lengths, scale)
            ctx.save_for_backward(tokens)
            ctx.V, ctx.lengths, ctx.scale = table.shape[0], lengths, scale
            ctx.mark_non_differentiable(status)
            return rows, status

        @staticmethod
        @once_differentiable
        def backward(ctx, grad_rows, _grad_status):
            (tokens,) = ctx.saved_tensors
            grad = binding.lfmmi_embed_tokens_backward(_rows_in_order(grad_rows), tokens, ctx.V, ctx.lengths,
                                                       ctx.scale)
            return grad, None, None, None

    return _EmbedTokens


_embed_cls = None


def embed_tokens(table, tokens, lengths=None, scale=1.0):
    """Rows of `table` [V, D] that `tokens` (int32 or int64 CUDA tensor [B, T] or [B]) name, times
    `scale`, differentiable in the table. Negative tokens and rows behind `lengths` (host ints [B]
    or None) give rows of 0 and no gradient. Returns (rows, status): tokens that are not below V
    give rows of NaN, a flag (4) in status and no gradient."""
    global _embed_cls
    if _embed_cls is None:
        _embed_cls = _embed_class()
    if lengths is not None:
        lengths = np.array(lengths, dtype=np.int32)  # (a copy: backward reads it)
    return _embed_cls.apply(_rows_in_order(table), tokens.contiguous(), lengths, float(scale))


def _dropout_class():
    import torch
    from torch.autograd.function import once_differentiable

    class _Dropout(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, p, seed, offset, step):
            ctx.draw = (p, seed, offset)
            ctx.save_for_backward(*([] if step is None else [step]))
            return binding.lfmmi_dropout(x, p, seed, offset, step)

        @staticmethod
        @once_differentiable
        def backward(ctx, grad):
            step = ctx.saved_tensors[0] if ctx.saved_tensors else None
            return binding.lfmmi_dropout(grad.contiguous(), *ctx.draw, step), None, None, None, None

    return _Dropout


_dropout_cls = None


def dropout(x, p, seed, offset=0, step=None):
    """Dropout of x [..., D], differentiable in x: a share p of the values becomes 0, the others are
    divided by 1 - p. What is kept follows from (seed, offset + step) and a value's row and
    column: give each call of a training run another offset. step: an int64 CUDA tensor of one
    value or None; backward reads it again, and refuses if it has been written since by an operation
    that torch knows of."""
    global _dropout_cls
    if _dropout_cls is None:
        _dropout_cls = _dropout_class()
    x = _rows_in_order(x)
    try:
        binding._flat_rows(x)
    except ValueError:
        x = x.contiguous()
    return _dropout_cls.apply(x, float(p), int(seed), int(offset), step)


def _copy_behind(out, rows, lengths):
    """The rows behind the lengths of a contiguous tensor [B, T, D] or [B, D], into their places in `out`."""
    import torch
    if rows.dim() == 2:
        out, rows = out[:, None], rows[:, None]
    T = rows.shape[1]
    places = [(out[b, n:], rows[b, n:]) for b, n in enumerate(lengths.tolist()) if n < T]
    if places:
        torch._foreach_copy_(*map(list, zip(*places)))   # (a launch for some hundred sequences)


def _norm_class():
    import torch
    from torch.autograd.function import once_differentiable

    class _AddRmsNorm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, residual, weight, eps, lengths, p, seed, offset, step):
            ctx.set_materialize_grads(False)  # what the loss does not use costs nothing
            r = binding.lfmmi_add_rms_norm(x, residual, weight, eps, lengths, p, seed, offset, step)
            ctx.draw, ctx.lengths, ctx.residual = (p, seed, offset), lengths, residual is not None
            ctx.sum_is_x = r.sum is x
            ctx.save_for_backward(r.sum, r.rstd, weight, step)
            return r.y, (r.sum.view_as(r.sum) if r.sum is x else r.sum)

        @staticmethod
        @once_differentiable
        def backward(ctx, grad_y, grad_sum):
            none = (None,) * 9
            if grad_y is None and grad_sum is None:
                return none
            total, rstd, weight, step = ctx.saved_tensors
            grad_y, grad_sum = (None if g is None else g.contiguous() for g in (grad_y, grad_sum))
            g = binding.lfmmi_add_rms_norm_backward(total, rstd, weight, grad_y, grad_sum,
                                                    ctx.lengths, *ctx.draw, step, residual=ctx.residual,
                                                    weight_grad=ctx.needs_input_grad[2])
            if ctx.sum_is_x and ctx.lengths is not None and grad_sum is not None and ctx.needs_input_grad[0]:
                _copy_behind(g.x, grad_sum, ctx.lengths)   # (x's own rows, which the forward call passes on)
            return (g.x, g.residual, g.weight) + none[3:]

    return _AddRmsNorm


_norm_cls = None


def add_rms_norm(x, residual=None, weight=None, eps=1e-6, lengths=None, p=0.0, seed=0, offset=0, step=None):
    """The end of a residual block: sum = residual + dropout(x) and y = sum / sqrt(mean(sum^2) + eps)
    * weight, rows [B, T, D] or [B, D], differentiable in x, residual and weight. Rows behind
    `lengths` (host ints [B] or None) give 0 and no gradient; p, seed, offset, step: as for
    dropout. Returns (y, sum): sum is what the next block adds to. Where nothing is added or dropped that
    is x itself, rows behind its lengths too, whose gradient is then x's. x and residual of two types
    are added in float32, as torch adds them, and y and sum are float32."""
    global _norm_cls
    if _norm_cls is None:
        _norm_cls = _norm_class()
    if lengths is not None:
        lengths = np.array(lengths, dtype=np.int32)  # (a copy: backward reads it)
    x = _rows_in_order(x)
    if residual is not None:
        residual = _rows_in_order(residual)
        if residual.dtype != x.dtype:   # (two of the three types: float32 holds every value of the others)
            if weight is not None and weight.dtype == x.dtype:
                weight = weight.float()
            x, residual = x.float(), residual.float()
    if weight is not None:
        weight = weight.contiguous()
    return _norm_cls.apply(x, residual, weight, float(eps), lengths, float(p), int(seed), int(offset), step)


def clip_grad_norm(parameters, max_norm):
    """Scales the gradients of `parameters` in place so that their norm, taken together, is at
    most max_norm, and returns the norm they had (a device tensor; nothing waits for it).
    Parameters without a gradient are passed over. A norm that is not finite makes
    all gradients 0: none of it reaches the weights, but an optimiser with momentum or
    weight decay still moves them unless its step is left out. Each gradient may be listed
    once."""
    grads = [p.grad for p in parameters if p.grad is not None]
    if not grads:
        raise ValueError("no parameter has a gradient")
    return binding.lfmmi_clip_grads(grads, max_norm)


def chain_loss(logits, lengths, num_graphs, den_graph, leak=1e-5, targets=None, target_weight=0.0):
    """Negative objective summed over the batch and divided by the number of frames
    (a scalar to minimise). Sequences flagged in `status` make it non-finite.

    targets: a frame alignment, an int32 or int64 CUDA tensor [B, T] of pdf-ids (negative: no
    target), whose frame log probabilities are added to the objective with target_weight; with a
    weight of 0 they are not looked at."""
    objf, _status = chain_objective(logits, lengths, num_graphs, den_graph, leak)
    frames = max(float(np.asarray(lengths, dtype=np.int64).sum()), 1.0)
    loss = -objf.sum() / frames
    if targets is not None and (not np.isscalar(target_weight) or target_weight != 0):
        logp, _entropy, _status = token_logprobs(logits, targets, lengths)
        loss = loss - logp.sum() * (target_weight / frames)
    return loss
