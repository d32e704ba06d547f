"""LF-MMI objective as a torch.autograd.Function on top of the C ABI (Eq. 2, Eq. 3), and
what a training step uses beside it: log probabilities of given tokens, and clipping of
gradients to a norm.

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
