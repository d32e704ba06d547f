"""What the operators on token log probabilities and on gradients refuse before they touch a
GPU, and the 64-bit forms that their kernels are compared with."""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest

from paper_2005_09824_amd import binding, chain
from tests import operators_oracle as oracle

INVALID, UNSUPPORTED = 1, 5
P = 4096  # an aligned address that nothing reads: every call here is refused


def _tokens(lengths=None, **kw):
    a = dict(logits=P, dtype=0, B=2, T=3, V=10, stride_b=30, stride_t=10, targets=P, target_bytes=8,
             scale=1.0, top_k=0, logp=P, entropy=P, stats=P, top_id=None, top_logp=None, status=P,
             workspace=None, workspace_bytes=0)
    a.update(kw)
    lens = None if lengths is None else np.asarray(lengths, np.int32)
    return binding.load_library().lfmmi_token_logprobs(
        a["logits"], a["dtype"], a["B"], a["T"], a["V"], a["stride_b"], a["stride_t"],
        None if lens is None else lens.ctypes.data, a["targets"], a["target_bytes"], a["scale"],
        a["top_k"], a["logp"], a["entropy"], a["stats"], a["top_id"], a["top_logp"], a["status"],
        a["workspace"], a["workspace_bytes"], None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(dtype=3), INVALID, "dtype"), (dict(dtype=-1), INVALID, "dtype"),
    (dict(B=-1), INVALID, "B and T"), (dict(T=-1), INVALID, "B and T"), (dict(V=0), INVALID, "V"),
    (dict(V=-5), INVALID, "V"), (dict(V=(1 << 30) + 1), UNSUPPORTED, "V"),
    (dict(B=1 << 16, T=1 << 15), UNSUPPORTED, "B * T"),
    (dict(stride_b=-1), INVALID, "strides"), (dict(stride_t=-1), INVALID, "strides"),
    (dict(stride_b=1 << 60), UNSUPPORTED, "strides"), (dict(stride_t=1 << 60), UNSUPPORTED, "strides"),
    (dict(scale=0.0), INVALID, "scale"), (dict(scale=-1.0), INVALID, "scale"),
    (dict(scale=float("nan")), INVALID, "scale"), (dict(scale=float("inf")), INVALID, "scale"),
    (dict(scale=1e7), INVALID, "scale"), (dict(target_bytes=2), INVALID, "target_bytes"),
    (dict(logits=None), INVALID, "logits"), (dict(logits=P + 2), INVALID, "aligned"),
    (dict(targets=P + 4), INVALID, "aligned"), (dict(dtype=1, logits=P + 1), INVALID, "aligned"),
    (dict(targets=None), INVALID, "logp"), (dict(top_k=-1), INVALID, "top_k"),
    (dict(top_k=11), INVALID, "top_k"), (dict(top_k=65, V=1000, stride_t=1000), UNSUPPORTED, "top_k"),
    (dict(lengths=[3, 4]), INVALID, "lengths[1]"), (dict(lengths=[-1, 0]), INVALID, "lengths[0]"),
])
def test_refused_token_calls(kw, code, text):
    assert _tokens(**kw) == code and text in binding.lfmmi_last_error(), binding.lfmmi_last_error()


def test_empty_token_calls_touch_nothing():
    assert _tokens(B=0) == 0 and _tokens(T=0) == 0 and _tokens(B=0, logits=None) == 0


def _backward(**kw):
    a = dict(logits=P, dtype=0, B=2, T=3, V=10, stride_b=30, stride_t=10, targets=P, target_bytes=4,
             scale=1.0, stats=P, entropy=P, grad_logp=P, grad_entropy=P, grad=1 << 20)
    a.update(kw)
    return binding.load_library().lfmmi_token_logprobs_backward(
        a["logits"], a["dtype"], a["B"], a["T"], a["V"], a["stride_b"], a["stride_t"], None,
        a["targets"], a["target_bytes"], a["scale"], a["stats"], a["entropy"], a["grad_logp"],
        a["grad_entropy"], a["grad"], None)


@pytest.mark.parametrize("kw,text", [
    (dict(dtype=9), "dtype"), (dict(V=0), "V"), (dict(scale=0.0), "scale"), (dict(logits=None), "logits"),
    (dict(targets=None), "targets"), (dict(entropy=None), "entropy"), (dict(stats=None), "stats"),
    (dict(grad=None), "grad"), (dict(grad=(1 << 20) + 2), "aligned"),
    (dict(grad=P + 4), "overlaps"), (dict(grad=P, stride_t=11, stride_b=33), "overlaps"),
    (dict(grad=P - 4 * 59), "overlaps"), (dict(grad=P, stride_b=40), "overlaps"),
])
def test_refused_backward_calls(kw, text):
    assert _backward(**kw) == INVALID and text in binding.lfmmi_last_error(), binding.lfmmi_last_error()


def test_workspace_sizes():
    lib = binding.load_library()
    n = ctypes.c_int64(-1)
    assert lib.lfmmi_token_logprobs_workspace(0, 2, 3, 10, 4, ctypes.byref(n)) == 0 and n.value == 0
    for args in ((7, 1, 1, 10, 0), (0, -1, 1, 10, 0), (0, 1, 1, 0, 0), (0, 1, 1, 10, 11), (0, 1, 1, 100, 65),
                 (0, 1, 1, 10, -1)):
        assert lib.lfmmi_token_logprobs_workspace(*args, ctypes.byref(n)) == INVALID
    assert lib.lfmmi_token_logprobs_workspace(0, 1, 1, 10, 0, None) == INVALID
    assert lib.lfmmi_token_logprobs_workspace(0, 1 << 16, 1 << 15, 10, 0, ctypes.byref(n)) == UNSUPPORTED


def _clip(n=2, grads=(P, 2 * P), counts=(10, 10), dtypes=(0, 0), outs=None, max_norm=1.0, norm=64 * P,
          workspace=128 * P, size=None, entry="clip"):
    lib = binding.load_library()
    arr = lambda t, v: None if v is None else (t * max(len(v), 1))(*v)
    g, c, d = arr(ctypes.c_void_p, grads), arr(ctypes.c_int64, counts), arr(ctypes.c_int32, dtypes)
    size = 16384 + 32 * (max(n, 0) + 1) if size is None else size
    if entry == "norm":
        return lib.lfmmi_grad_norm(n, g, c, d, norm, workspace, size, None)
    return lib.lfmmi_clip_grads(n, g, arr(ctypes.c_void_p, outs), c, d, max_norm, norm, workspace, size, None)


@pytest.mark.parametrize("kw,code,text", [
    (dict(n=-1), INVALID, "n must"), (dict(norm=None), INVALID, "norm"), (dict(grads=None), INVALID, "null"),
    (dict(counts=None), INVALID, "null"), (dict(dtypes=None), INVALID, "null"),
    (dict(workspace=None), INVALID, "workspace"), (dict(workspace=P + 8), INVALID, "workspace"),
    (dict(size=100), INVALID, "workspace"), (dict(dtypes=(0, 5)), INVALID, "dtype"),
    (dict(counts=(1, -1)), INVALID, "counts"), (dict(counts=(1, (1 << 36) + 1)), UNSUPPORTED, "count"),
    (dict(grads=(P, None)), INVALID, "grads[1]"), (dict(grads=(P, 2 * P + 2)), INVALID, "aligned"),
])
@pytest.mark.parametrize("entry", ["clip", "norm"])
def test_refused_gradient_calls(kw, code, text, entry):
    assert _clip(entry=entry, **kw) == code and text in binding.lfmmi_last_error(), binding.lfmmi_last_error()


@pytest.mark.parametrize("kw,text", [
    (dict(max_norm=-1.0), "max_norm"), (dict(max_norm=float("nan")), "max_norm"),
    (dict(outs=(P, None)), "outs[1]"), (dict(outs=(P, 2 * P + 1)), "aligned"),
    (dict(grads=(P, P)), "listed twice"), (dict(grads=(P, P + 36)), "overlaps"),
    (dict(grads=(P + 36, P)), "overlaps"), (dict(outs=(2 * P, P)), "overlaps"),
    (dict(outs=(8 * P, 8 * P + 4)), "overlaps"), (dict(outs=(P + 4, 8 * P)), "overlaps"),
    (dict(grads=(P, P + 4), outs=(P, 8 * P)), "overlaps"),
])
def test_refused_clipping(kw, text):
    assert _clip(**kw) == INVALID and text in binding.lfmmi_last_error(), binding.lfmmi_last_error()


def test_binding_refuses_what_is_not_on_a_gpu():
    import torch
    x = torch.zeros((3, 5))
    t = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        binding.lfmmi_token_logprobs(x, t)
    with pytest.raises(ValueError):
        binding.lfmmi_token_logprobs_backward(x, t, torch.zeros((3, 2)), None, torch.zeros(3))
    with pytest.raises(ValueError):
        chain.token_logprobs(x, t)
    for call in (binding.lfmmi_grad_norm, lambda g: binding.lfmmi_clip_grads(g, 1.0)):
        with pytest.raises(ValueError):
            call([x])
        with pytest.raises(ValueError):
            call([])
    with pytest.raises(ValueError):
        chain.clip_grad_norm([torch.nn.Parameter(x)], 1.0)


def test_dense_layouts():
    import torch
    x = torch.zeros((4, 6, 5))
    for y in (x, x.permute(2, 0, 1), x[1:3], torch.zeros(()), x[:1, :1, :1],
              torch.zeros((2, 0, 3)).permute(2, 1, 0), torch.zeros((5, 1, 7)).transpose(0, 2)):
        assert binding._dense(y)
    for y in (x[:, ::2], x[:, :, :4], x.view(-1)[::5], x[:, :1].permute(1, 0, 2), x[:, :1].expand(4, 3, 5),
              torch.zeros(9).as_strided((4, 3), (1, 1))):
        assert not binding._dense(y)


def test_oracle_gradient_against_differences():
    rng = np.random.default_rng(0)
    x = rng.normal(0, 2, (5, 9))
    t = rng.integers(0, 9, 5)
    g, h = rng.normal(0, 1, 5), rng.normal(0, 1, 5)
    r = oracle.rows(x, t, np.ones(5, bool), 0.8, 3)
    grad = oracle.grads(r, t, np.ones(5, bool), 0.8, g, h)
    for n in range(5):
        for i in range(9):
            e = np.zeros_like(x)
            e[n, i] = 1e-6
            diff = (oracle.loss(x + e, t, 0.8, g, h) - oracle.loss(x - e, t, 0.8, g, h)) / 2e-6
            assert abs(diff - grad[n, i]) < 1e-8


def test_oracle_rows_by_hand():
    # two tokens of equal weight and one that is masked
    r = oracle.rows([[1.0, -np.inf, 1.0]], np.array([2]), [True], 1.0, 3)
    assert abs(r["logp"][0] + np.log(2)) < 1e-15 and abs(r["entropy"][0] - np.log(2)) < 1e-15
    assert r["top_id"].tolist() == [[0, 2, 1]] and r["top_logp"][0, 2] == -np.inf


class _OnGpu:
    """What the binding asks of a tensor of `shape` on a GPU."""
    is_cuda = True

    def __init__(self, shape):
        import torch
        t = torch.empty(1, dtype=torch.float32).expand(shape)
        self.dtype, self.shape, self.device = t.dtype, t.shape, t.device
        self.dim, self.stride = t.dim, lambda: t.stride()[:-1] + (1,)


@pytest.mark.parametrize("shape", [((1 << 32) + 5, 4), (1 << 31, 4), (3, (1 << 32) + 7), (2, (1 << 32) + 1, 4),
                                   ((1 << 32) + 1, 2, 4), (1 << 20, 1 << 20, 4), (2, 3, 1 << 33)])
def test_sizes_beyond_the_libraries_types_are_refused(shape):
    # (a size that is passed on as its lowest 32 bits scores the first rows or columns alone)
    with pytest.raises(ValueError, match="too many rows or columns"):
        binding._logit_rows(_OnGpu(shape), None, None)
    assert binding._logit_rows(_OnGpu((5, 3, 4)), None, None)[:4] == (0, 5, 3, 4)


@pytest.mark.parametrize("kw", [
    dict(norm=P + 36), dict(norm=2 * P), dict(workspace=P), dict(grads=(P, 40 * P), workspace=40 * P - 16384), dict(workspace=2 * P + 32),
    dict(norm=128 * P + 16), dict(norm=128 * P + 16384 + 32 * 3 - 4), dict(norm=128 * P),
    dict(grads=(P, 128 * P + 16384 + 92)), dict(n=1, grads=(128 * P - 8,), counts=(3,), dtypes=(0,)),
])
@pytest.mark.parametrize("entry", ["clip", "norm"])
def test_norm_and_workspace_overlap_nothing(kw, entry):
    # (a table of addresses in the workspace, scaled like a gradient, would send writes anywhere)
    assert _clip(entry=entry, **kw) == INVALID and "norm or workspace overlaps" in binding.lfmmi_last_error()


@pytest.mark.parametrize("outs", [(64 * P - 36, 8 * P), (64 * P, 8 * P), (8 * P, 128 * P + 16384 + 32 * 3 - 4),
                                  (8 * P, 128 * P - 36)])
def test_outputs_overlap_neither_norm_nor_workspace(outs):
    assert _clip(outs=outs) == INVALID and "norm or workspace overlaps" in binding.lfmmi_last_error()


def test_workspace_of_rows_that_the_call_refuses():
    lib = binding.load_library()
    n = ctypes.c_int64(-1)
    for V in ((1 << 30) + 1, (1 << 31) - 1):
        assert lib.lfmmi_token_logprobs_workspace(1, 1, 1, V, 0, ctypes.byref(n)) == UNSUPPORTED, n.value
        assert "V" in binding.lfmmi_last_error()
    assert lib.lfmmi_token_logprobs_workspace(1, 1, 1, 1 << 30, 0, ctypes.byref(n)) == 0 and n.value > 0


def test_an_alignment_of_no_weight_is_not_scored(monkeypatch):
    # (0 times the log probability of a token that is masked out would be NaN)
    import torch
    objf = torch.tensor([-3.0, -5.0], requires_grad=True)
    monkeypatch.setattr(chain, "chain_objective", lambda *a: (objf, None))
    scored = []

    def logprobs(logits, targets, lengths):
        scored.append(targets)
        return torch.tensor([[0.0, -float("inf")], [-1.0, -2.0]]), None, None

    monkeypatch.setattr(chain, "token_logprobs", logprobs)
    targets = torch.zeros((2, 2), dtype=torch.int64)
    for weight in (0, 0.0, -0.0, np.float32(0)):
        assert float(chain.chain_loss(None, [2, 2], None, None, 1e-5, targets, weight).detach()) == 2.0
    assert float(chain.chain_loss(None, [2, 2], None, None, 1e-5, targets).detach()) == 2.0 and not scored
    assert float(chain.chain_loss(None, [2, 2], None, None, 1e-5, targets, 0.5).detach()) == float("inf")
    assert float(chain.chain_loss(None, [2, 2], None, None, 1e-5, targets, torch.tensor(0.5)).detach()) == float("inf")
    assert len(scored) == 2


def test_outputs_laid_out_as_their_gradients_are(monkeypatch):
    # strides of dimensions of one entry say nothing
    import torch
    described = binding._described
    monkeypatch.setattr(binding, "_described", lambda t: ([0] * len(t),) + described(t)[1:])  # as on a GPU
    last = dict(memory_format=torch.channels_last)
    conv, depthwise = torch.zeros((4, 8, 5, 5)).to(**last), torch.zeros((8, 1, 3, 3)).to(**last)
    assert depthwise.is_contiguous() and depthwise.stride() != (9, 9, 3, 1)
    grads = [conv, depthwise, torch.zeros((5, 1, 7)).transpose(0, 2), torch.zeros((3, 4))]
    out = [torch.zeros((4, 8, 5, 5)).to(**last), torch.zeros((8, 1, 3, 3)), torch.zeros((5, 7)).t().unsqueeze(1),
           torch.zeros(12)]
    assert out[2].stride() != grads[2].stride()
    pointers, outs, counts, codes = binding._grad_arrays(grads, out)
    assert list(outs) == [o.data_ptr() for o in out] and list(counts) == [g.numel() for g in grads]
    for i, bad in ((0, torch.zeros((4, 8, 5, 5))), (1, torch.zeros((8, 1, 3, 3)).transpose(2, 3)), (3, torch.zeros((4, 3)).t()),
                   (2, torch.zeros((7, 1, 5))), (3, torch.zeros(11)), (0, torch.zeros((8, 4, 5, 5)).to(**last))):
        with pytest.raises(ValueError, match="output tensor"):
            binding._grad_arrays(grads, [bad if j == i else o for j, o in enumerate(out)])


def test_a_call_that_runs_out_of_host_memory_says_so():
    # in a process of its own, with 200 MB more than the lists take: the check of overlaps would
    # need 960 MB for them
    code = """if True:
        import resource
        import numpy as np
        from paper_2005_09824_amd import binding
        lib = binding.load_library()
        assert lib.lfmmi_grad_norm(-1, None, None, None, None, None, 0, None) == 1   # (a text that is there before)
        n = 20000000
        pointers, counts, codes = np.zeros(n, np.uint64), np.zeros(n, np.int64), np.zeros(n, np.int32)
        for a in (pointers, counts, codes):
            a.fill(0)
        used = int(open("/proc/self/statm").read().split()[0]) * 4096
        resource.setrlimit(resource.RLIMIT_AS, (used + (200 << 20), resource.RLIM_INFINITY))
        code = lib.lfmmi_clip_grads(n, pointers.ctypes.data, None, counts.ctypes.data, codes.ctypes.data, 1.0, 4096,
                                    1 << 40, 16384 + 32 * (n + 1), None)
        print(code, binding.lfmmi_last_error())
    """
    run = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=100,
                         cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert run.stdout.strip() == "3 host allocation failed", (run.stdout, run.stderr)
