"""Performance cases of the layer operators: what a training step or a served
request has them compute, from one token to thousands.

Kinds
-----
* ``linear``    O = act(F X + bias) + residual, one matrix product with the rest
                in its epilogue (``linear``); with ``pre`` the pre-activation is
                kept for the backward pass.
* ``backward``  its gradients: dX, dF and dbias from dO (``linear_backward``).
* ``clip``      the norm of all gradients together, and the gradients scaled to
                at most ``max_norm`` (``clip_grad_norm`` into buffers of the
                optimizer); ``only`` asks for the norm alone (``grad_norm``).

F is (kn, ci), X is (ci, t) and O is (kn, t), the convolution's names: kn
outputs, ci inputs, t tokens (or images).  X and O are stored with the leftmost
index fastest; ``order`` says which index of F is: "kn" as the convolution's
filters, "ci" as a row-major weight seen through a view.

Inputs are drawn on the GPU from the seed: activations and incoming gradients
standard normal, weights normal with variance 1 / ci, gradients normal with a
norm well above ``max_norm``.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_MAX_NORM = 1.0


def _linear(name, kn, ci, t, dtype, order, act, bias, residual, pre):
    return {"name": name, "kind": "linear", "kn": kn, "ci": ci, "t": t, "dtype": dtype, "order": order, "act": act,
            "bias": bias, "residual": residual, "pre": pre}


def _backward(name, kn, ci, t, dtype, order, act):
    return {"name": name, "kind": "backward", "kn": kn, "ci": ci, "t": t, "dtype": dtype, "order": order, "act": act}


def listed():
    return [
        # -- one layer, forward -------------------------------------------------
        # one token of a served model: a square projection back onto the residual
        # stream, bound by one read of its weights
        _linear("linear_t1_4096x4096", 4096, 4096, 1, "bf16", "ci", "none", True, True, False),
        # eight requests decoded together through a wide layer, filters stored as
        # the convolution stores them
        _linear("linear_t8_16384x4096_gelu", 16384, 4096, 8, "bf16", "kn", "gelu", True, False, False),
        # the fully connected layer behind a convolution stack, at the
        # benchmark's batch of 80 images, single precision as the convolution
        _linear("linear_t80_4096x9216_relu", 4096, 9216, 80, "f32", "kn", "relu", True, False, False),
        # a short prompt into a thousand classes
        _linear("linear_t300_1000x4096", 1000, 4096, 300, "f16", "ci", "none", True, False, False),
        # ragged everywhere: no size is a multiple of anything
        _linear("linear_t2047_1535x1001_silu", 1535, 1001, 2047, "f16", "ci", "silu", True, True, False),
        # the largest: a training step's widening layer over 8192 tokens, its
        # pre-activation kept for the backward pass
        _linear("linear_t8192_16384x4096_gelu", 16384, 4096, 8192, "bf16", "ci", "gelu", True, False, True),
        # -- its gradients --------------------------------------------------------
        # the classifier of the same stack, trained on 80 images at a time
        _backward("backward_t80_1000x4096", 1000, 4096, 80, "f32", "kn", "none"),
        # a small ragged layer behind a GELU
        _backward("backward_t777_1001x515_gelu", 1001, 515, 777, "f16", "ci", "gelu"),
        # the largest: the narrowing layer of the same training step
        _backward("backward_t8192_4096x16384", 4096, 16384, 8192, "bf16", "ci", "none"),
        # -- norm and clipping ------------------------------------------------------
        # a small network's gradients: launches and latency are everything
        {"name": "clip_8_small", "kind": "clip", "count": 8, "total": 600_001, "dtype": "f32", "only": False},
        # a model's worth of tensors, sizes from a few values to millions
        {"name": "clip_200_ragged", "kind": "clip", "count": 200, "total": 90_000_017, "dtype": "bf16", "only": False},
        # the largest: single-precision gradients of the whole model
        {"name": "clip_48_large", "kind": "clip", "count": 48, "total": 400_000_000, "dtype": "f32", "only": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng):
    """A layer's width: half of them multiples of 64, the rest as they come."""
    n = _log_int(rng, 64, 16384)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "backward", "backward", "clip", "clip"])
    if kind == "clip":
        return {"kind": kind, "count": _log_int(rng, 1, 300), "total": _log_int(rng, 10_000, 300_000_000),
                "dtype": rng.choice(["f32", "bf16", "f16"]), "only": rng.random() < 0.3}
    while True:
        c = {"kind": kind, "kn": _width(rng), "ci": _width(rng), "t": _log_int(rng, 1, 8192),
             "dtype": rng.choice(["f32", "bf16", "bf16", "f16"]), "order": rng.choice(["kn", "ci"]),
             "act": rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"])}
        if kind == "linear":
            c["bias"], c["residual"] = rng.random() < 0.7, rng.random() < 0.5
            c["pre"] = c["act"] != "none" and rng.random() < 0.5
        # single precision runs at a sixteenth of the 16-bit types' rate
        if work(c)["flops"] < (1e12 if c["dtype"] != "f32" else 1e11):
            return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype, scale=1.0):
    """Normal values, (d0, d1) stored with d0 fastest."""
    x = torch.randn(tuple(reversed(shape)), generator=g, device="cuda", dtype=dtype)
    if scale != 1.0:
        x *= scale
    return x.t() if len(shape) == 2 else x


def _sizes(case):
    """The tensors' sizes: spread over their logarithm, `total` in all."""
    rng = random.Random(case["count"] * 1_000_003 + case["total"])
    w = [math.exp(rng.uniform(0.0, 7.0)) for _ in range(case["count"])]
    sizes = [max(1, int(case["total"] * v / sum(w))) for v in w]
    sizes[0] = max(1, sizes[0] + case["total"] - sum(sizes))
    return sizes


def prepare(case, seed):
    g = _gen(seed)
    dtype = _DTYPES[case["dtype"]]
    if case["kind"] == "clip":
        sizes = _sizes(case)
        grads = [_normal(g, (n,), dtype, 0.05) for n in sizes]
        if case["only"]:
            return {"case": case, "grads": grads}
        # one buffer for the scaled gradients, every tensor's part 64 values aligned
        at, ends = 0, []
        for n in sizes:
            ends.append((at, n))
            at += (n + 63) // 64 * 64
        flat = torch.zeros(at, dtype=dtype, device="cuda")
        return {"case": case, "grads": grads, "flat": flat, "out": [flat[a:a + n] for a, n in ends]}
    kn, ci, t = case["kn"], case["ci"], case["t"]
    F = _normal(g, (kn, ci), dtype, ci ** -0.5) if case["order"] == "kn" else _normal(g, (ci, kn), dtype, ci ** -0.5).t()
    s = {"case": case, "F": F, "X": _normal(g, (ci, t), dtype)}
    if case["kind"] == "linear":
        s["bias"] = _normal(g, (kn,), dtype, 0.1) if case["bias"] else None
        s["residual"] = _normal(g, (kn, t), dtype) if case["residual"] else None
    else:
        s["dO"] = _normal(g, (kn, t), dtype)
        s["pre"] = _normal(g, (kn, t), dtype) if case["act"] != "none" else None
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        th = torch.tanh(a * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + th) + 0.5 * z * (1 - th * th) * a * (1 + 3 * 0.044715 * z * z)
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s))


def _plain_linear(s):
    c, dtype = s["case"], s["X"].dtype
    z = (s["X"].t().float() @ s["F"].t().float()).t()
    if s["bias"] is not None:
        z = z + s["bias"].float()[:, None]
    o = _act(z, c["act"])
    if s["residual"] is not None:
        o = o + s["residual"].float()
    return (o.to(dtype), z.to(dtype)) if c["pre"] else o.to(dtype)


def _plain_backward(s):
    c, dtype = s["case"], s["X"].dtype
    dz = s["dO"].float()
    if c["act"] != "none":
        dz = dz * _act_slope(s["pre"].float(), c["act"])
    dX = (dz.t() @ s["F"].float()).t()
    dF = (s["X"].float() @ dz.t()).t()
    return dX.to(dtype), dF.to(dtype), dz.sum(1).to(dtype)


def _plain_clip(s):
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    if s["case"]["only"]:
        return norm
    scale = (_MAX_NORM / norm).clamp_max(1.0)
    _ = [o.copy_(g.float() * scale) for g, o in zip(s["grads"], s["out"])]
    return norm, s["flat"]


def run(s):
    c = s["case"]
    if not own:
        return {"linear": _plain_linear, "backward": _plain_backward, "clip": _plain_clip}[c["kind"]](s)
    import paper_2005_06410_amd as lt
    if c["kind"] == "linear":
        return lt.linear(s["F"], s["X"], bias=s["bias"], activation=c["act"], residual=s["residual"],
                         keep_pre=c["pre"])
    if c["kind"] == "backward":
        return lt.linear_backward(s["F"], s["X"], s["dO"], pre=s["pre"], activation=c["act"])
    if c["only"]:
        return lt.grad_norm(s["grads"])
    return lt.clip_grad_norm(s["grads"], _MAX_NORM, out=s["out"]), s["flat"]


def work(case):
    size = _BYTES[case["dtype"]]
    if case["kind"] == "clip":
        n = case["total"]
        return {"bytes": float(size * n * (1 if case["only"] else 2)), "flops": float(n * (2 if case["only"] else 3))}
    kn, ci, t = case["kn"], case["ci"], case["t"]
    if case["kind"] == "linear":
        values = kn * ci + ci * t + kn * t * (1 + bool(case["residual"]) + bool(case["pre"])) + (kn if case["bias"] else 0)
        return {"bytes": float(size * values), "flops": 2.0 * kn * ci * t}
    values = 2 * (kn * ci + ci * t) + kn * t * (2 if case["act"] != "none" else 1) + kn
    return {"bytes": float(size * values), "flops": 4.0 * kn * ci * t}


# ---------------------------------------------------------------------------
# the definition, in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "clip":
        total = 0.0
        for g in s["grads"]:
            v = g.double()
            total += float((v * v).sum())
        norm = math.sqrt(total)
        answer = torch.tensor(norm, dtype=torch.float64)
        if case["only"]:
            return answer
        flat = torch.zeros(s["flat"].numel(), dtype=torch.float64, device="cuda")
        for g, o in zip(s["grads"], s["out"]):
            flat[o.storage_offset():o.storage_offset() + o.numel()] = g.double() * min(1.0, _MAX_NORM / norm)
        return answer, flat
    F, X = s["F"].double(), s["X"].double()
    phi = lambda z: 0.5 * torch.erfc(-z / math.sqrt(2.0))                              # noqa: E731  normal distribution
    density = lambda z: torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)                 # noqa: E731
    inner = lambda z: math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)                 # noqa: E731
    logistic = lambda z: 1 / (1 + torch.exp(-z))                                       # noqa: E731
    # 0.5 (1 + tanh u) is the logistic function of 2u
    value = {"none": lambda z: z, "relu": lambda z: torch.where(z > 0, z, torch.zeros_like(z)),
             "gelu": lambda z: z * phi(z), "gelu_tanh": lambda z: z * logistic(2 * inner(z)),
             "silu": lambda z: z * logistic(z)}
    slope = {"none": torch.ones_like, "relu": lambda z: torch.where(z > 0, 1.0, 0.0).double(),
             "gelu": lambda z: phi(z) + z * density(z),
             "gelu_tanh": lambda z: (logistic(2 * inner(z)) + z * 2 * logistic(2 * inner(z)) * logistic(-2 * inner(z))
                                     * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z ** 2)),
             "silu": lambda z: logistic(z) + z * logistic(z) * logistic(-z)}
    if case["kind"] == "linear":
        z = torch.matmul(F, X)
        if s["bias"] is not None:
            z = z + s["bias"].double().unsqueeze(1)
        o = value[case["act"]](z)
        if s["residual"] is not None:
            o = o + s["residual"].double()
        return (o, z) if case["pre"] else o
    dz = s["dO"].double()
    if case["act"] != "none":
        dz = dz * slope[case["act"]](s["pre"].double())
    return torch.matmul(F.t(), dz), torch.matmul(dz, X.t()), dz.sum(dim=1)
