"""Performance cases of the operators that end and normalise a network: the loss of
a classifier or a language model over a large vocabulary without its logits in
memory, distillation from a teacher's largest logits, and group norm with an
activation behind a convolution.

Kinds
-----
* ``loss``     softmax cross entropy of Z = F X + bias with one label a token
               (``linear_cross_entropy``); with ``train`` its gradients, too
               (``linear_cross_entropy_backward``).
* ``distill``  T^2 KL(teacher || softmax(Z / T)), the teacher given by its k largest
               logits a token (``linear_distill``, ``linear_distill_backward``).
* ``norm``     group norm of channels-last images with an activation
               (``group_norm``, ``group_norm_backward``).

F is (kn, ci), X is (ci, t), the layer's names: kn classes or words, ci features, t
tokens (or images).  X is stored with the leftmost index fastest; ``order`` says which
index of F is: "kn" as the convolution's filters, "ci" as a row-major weight seen
through a view.  The norm's input is (c, h, w, b), a convolution's output, leftmost
index fastest.

Inputs are drawn on the GPU from the seed.  Features are normal with a share of the
right class's weights added, so that logits spread over a range of about 2.5 and the
right one is often among the largest; a tenth of the tokens are padding (label -100);
gradients arrive as the mean's 1 / t, for fp16 times a loss scale of 1024.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_SPREAD = 2.5
_IGNORE = -100
_EPS = 1e-5


def _loss(name, kn, ci, t, dtype, order, bias, train):
    return {"name": name, "kind": "loss", "kn": kn, "ci": ci, "t": t, "dtype": dtype, "order": order, "bias": bias,
            "train": train}


def _distill(name, kn, ci, t, k, temperature, dtype, order, bias, train):
    return {"name": name, "kind": "distill", "kn": kn, "ci": ci, "t": t, "k": k, "temperature": temperature,
            "dtype": dtype, "order": order, "bias": bias, "train": train}


def _norm(name, c, groups, h, w, b, dtype, act, train):
    return {"name": name, "kind": "norm", "c": c, "groups": groups, "h": h, "w": w, "b": b, "dtype": dtype, "act": act,
            "train": train}


def listed():
    return [
        # -- cross entropy over a vocabulary --------------------------------------
        # one token scored while a model is served: one read of the head's weights
        _loss("loss_t1_32000x4096", 32000, 4096, 1, "bf16", "ci", False, False),
        # the classifier of a convolution stack, trained on the benchmark's 80 images
        _loss("loss_t80_1000x4096_train", 1000, 4096, 80, "f32", "kn", True, True),
        # ragged everywhere: no size is a multiple of anything
        _loss("loss_t777_10007x1001_train", 10007, 1001, 777, "f16", "ci", True, True),
        # the largest: a training step's head over 8192 tokens
        _loss("loss_t8192_131072x4096_train", 131072, 4096, 8192, "bf16", "ci", False, True),
        # -- distillation -----------------------------------------------------------
        # a validation batch of a small student: launches and latency
        _distill("distill_t33_1000x512_k5", 1000, 512, 33, 5, 4.0, "f32", "kn", True, False),
        # ragged everywhere, weights stored as the convolution stores them
        _distill("distill_t300_50021x777_k17_train", 50021, 777, 300, 17, 2.0, "f16", "kn", True, True),
        # a student's training step from 64 stored logits a token
        _distill("distill_t4096_32000x4096_k64_train", 32000, 4096, 4096, 64, 1.0, "bf16", "ci", False, True),
        # -- group norm ---------------------------------------------------------------
        # one image behind a small convolution, served
        _norm("norm_c384_13x13_b1", 384, 32, 13, 13, 1, "f32", "relu", False),
        # the same stack's larger maps, trained on 80 images
        _norm("norm_c256_27x27_b80_train", 256, 32, 27, 27, 80, "f32", "relu", True),
        # ragged: ten channels a group, odd maps
        _norm("norm_c90_31x45_b7_train", 90, 9, 31, 45, 7, "f16", "silu", True),
        # no map at all: the features of each token in groups
        _norm("norm_c1000_t4001_train", 1000, 8, 1, 1, 4001, "bf16", "gelu", True),
        # the largest: maps of an image generator
        _norm("norm_c128_256x256_b16_train", 128, 32, 256, 256, 16, "bf16", "silu", True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: half of them multiples of 64, the rest as they come."""
    n = _log_int(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


def draw(rng):
    kind = rng.choice(["loss", "loss", "distill", "distill", "norm", "norm"])
    if kind == "norm":
        while True:
            groups = _log_int(rng, 1, 64)
            c = {"kind": kind, "c": groups * _log_int(rng, 1, 64), "groups": groups, "h": _log_int(rng, 1, 256),
                 "w": _log_int(rng, 1, 256), "b": _log_int(rng, 1, 128), "dtype": rng.choice(["f32", "bf16", "f16"]),
                 "act": rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), "train": rng.random() < 0.7}
            # a channel that is a group of its own needs a map to vary over
            if 100_000 < c["c"] * c["h"] * c["w"] * c["b"] < 100_000_000 and c["c"] // groups * c["h"] * c["w"] >= 16:
                return c
    while True:
        c = {"kind": kind, "kn": _width(rng, 1000, 131072), "ci": _width(rng, 64, 8192), "t": _log_int(rng, 1, 8192),
             "dtype": rng.choice(["f32", "bf16", "bf16", "f16"]), "order": rng.choice(["kn", "ci"]),
             "bias": rng.random() < 0.5, "train": rng.random() < 0.7}
        if kind == "distill":
            c["k"], c["temperature"] = _log_int(rng, 1, 128), rng.choice([1.0, 2.0, 4.0])
        # single precision runs at a sixteenth of the 16-bit types' rate
        if work(c)["flops"] < (8e12 if c["dtype"] != "f32" else 5e11) and c["kn"] * c["ci"] < 600_000_000:
            return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, dtype, scale=1.0):
    """Normal values, stored with the leftmost index fastest."""
    x = torch.randn(tuple(reversed(shape)), generator=g, device="cuda", dtype=dtype)
    if scale != 1.0:
        x *= scale
    return x.permute(*reversed(range(len(shape))))


def _prepare_norm(case, g, dtype):
    c, shape = case["c"], (case["c"], case["h"], case["w"], case["b"])
    # every channel has an offset and a scale of its own, as behind a convolution
    x = _normal(g, shape, dtype)
    scale = (_normal(g, (c,), dtype, 0.3) + 1).view(c, 1, 1, 1)
    offset = _normal(g, (c,), dtype, 0.5).view(c, 1, 1, 1)
    s = {"case": case, "x": x.mul_(scale).add_(offset), "weight": 1 + _normal(g, (c,), dtype, 0.2),
         "bias": _normal(g, (c,), dtype, 0.2)}
    if case["train"]:
        s["dO"] = _normal(g, shape, dtype)
    return s


def prepare(case, seed):
    g = _gen(seed)
    dtype = _DTYPES[case["dtype"]]
    if case["kind"] == "norm":
        return _prepare_norm(case, g, dtype)
    kn, ci, t = case["kn"], case["ci"], case["t"]
    scale = _SPREAD * ci ** -0.5
    F = _normal(g, (kn, ci), dtype, scale) if case["order"] == "kn" else _normal(g, (ci, kn), dtype, scale).t()
    s = {"case": case, "F": F, "bias": _normal(g, (kn,), dtype, 0.5) if case["bias"] else None}
    right = torch.randint(0, kn, (t,), generator=g, device="cuda")
    x = torch.randn(t, ci, generator=g, device="cuda", dtype=dtype)
    share = torch.rand(t, 1, generator=g, device="cuda").to(dtype)
    s["X"] = (x + share * F[right]).t()
    mean = (1024.0 if case["dtype"] == "f16" else 1.0) / t
    s["dloss"] = torch.full((t,), mean, dtype=torch.float32, device="cuda")
    if case["kind"] == "loss":
        pad = torch.rand(t, generator=g, device="cuda") < 0.1
        s["labels"] = torch.where(pad & (torch.arange(t, device="cuda") > 0), _IGNORE, right)
        return s
    # k different words a token, the right one first, the teacher's logits from the
    # largest down
    k = case["k"]
    step = torch.randint(1, max(2, kn // k), (t, k), generator=g, device="cuda")
    step[:, 0] = 0
    index = (right[:, None] + step.cumsum(1)) % kn
    order = torch.rand(t, k, generator=g, device="cuda")
    order[:, 0] = -1
    top = torch.randn(t, k, generator=g, device="cuda").mul_(2).sort(dim=1, descending=True)[0]
    s["index"] = index.gather(1, order.argsort(dim=1)).t()
    s["top"] = top.to(dtype).t()
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
    if act == "none":
        return torch.ones_like(z)
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


def _plain_logits(s):
    """Z^T and its logsumexp, (t, kn) and (t, 1); with a temperature, of Z / T."""
    z = s["X"].t().float() @ s["F"].t().float()
    if s["bias"] is not None:
        z += s["bias"].float()
    if s["case"]["kind"] == "distill":
        z /= s["case"]["temperature"]
    top = z.max(dim=1, keepdim=True)[0]
    return z, top + torch.log(torch.exp(z - top).sum(dim=1, keepdim=True))


def _plain_gradients(s, dz):
    """dX, dF and dbias of dZ^T (t, kn), rounded once."""
    dtype = s["X"].dtype
    dX = (dz @ s["F"].float()).t()
    dF = dz.t() @ s["X"].t().float()
    return dX.to(dtype), dF.to(dtype), dz.sum(0).to(dtype)


def _plain_loss(s):
    z, lse = _plain_logits(s)
    labels = s["labels"]
    keep = labels != _IGNORE
    at = torch.where(keep, labels, 0)[:, None]
    loss = torch.where(keep, (lse - z.gather(1, at))[:, 0], 0.0)
    if not s["case"]["train"]:
        return loss, lse[:, 0]
    dz = torch.exp(z - lse)
    dz.scatter_add_(1, at, torch.full_like(lse, -1.0))
    dz *= (s["dloss"] * keep)[:, None]
    return (loss, lse[:, 0]) + _plain_gradients(s, dz)


def _plain_distill(s):
    temperature = s["case"]["temperature"]
    z, lse = _plain_logits(s)
    index, top = s["index"].t(), s["top"].t().float() / temperature
    best = top.max(dim=1, keepdim=True)[0]
    e = torch.exp(top - best)
    q = e / e.sum(dim=1, keepdim=True)
    log_q = top - best - torch.log(e.sum(dim=1, keepdim=True))
    loss = temperature * temperature * (q * (log_q - (z.gather(1, index) - lse))).sum(1)
    if not s["case"]["train"]:
        return loss, lse[:, 0]
    dz = torch.exp(z - lse)
    dz.scatter_add_(1, index, -q)
    dz *= (s["dloss"] * temperature)[:, None]
    return (loss, lse[:, 0]) + _plain_gradients(s, dz)


def _plain_norm(s):
    case, dtype = s["case"], s["x"].dtype
    g, b, s_ = case["groups"], case["b"], case["h"] * case["w"]
    per = case["c"] // g
    x = s["x"].permute(3, 2, 1, 0).reshape(b, s_, g, per).float()
    weight, bias = s["weight"].float().view(g, per), s["bias"].float().view(g, per)
    mean = x.mean(dim=(1, 3), keepdim=True)
    rstd = torch.rsqrt((x - mean).square().mean(dim=(1, 3), keepdim=True) + _EPS)
    xhat = (x - mean) * rstd
    z = xhat * weight + bias

    def shaped(v):
        return v.to(dtype).view(b, case["w"], case["h"], case["c"]).permute(3, 2, 1, 0)

    out = (shaped(_act(z, case["act"])), mean.view(b, g).t(), rstd.view(b, g).t())
    if not case["train"]:
        return out
    dz = s["dO"].permute(3, 2, 1, 0).reshape(b, s_, g, per).float() * _act_slope(z, case["act"])
    dxhat = dz * weight
    dx = rstd * (dxhat - dxhat.mean(dim=(1, 3), keepdim=True) - xhat * (dxhat * xhat).mean(dim=(1, 3), keepdim=True))
    return out + (shaped(dx), (dz * xhat).sum(dim=(0, 1)).view(-1).to(dtype), dz.sum(dim=(0, 1)).view(-1).to(dtype))


def run(s):
    case = s["case"]
    if not own:
        return {"loss": _plain_loss, "distill": _plain_distill, "norm": _plain_norm}[case["kind"]](s)
    import paper_2005_06410_amd as lt
    if case["kind"] == "norm":
        out = lt.group_norm(s["x"], case["groups"], s["weight"], s["bias"], eps=_EPS, activation=case["act"])
        if not case["train"]:
            return out
        return out + lt.group_norm_backward(s["x"], s["dO"], case["groups"], out[1], out[2], s["weight"], s["bias"],
                                            activation=case["act"])
    if case["kind"] == "loss":
        loss, lse = lt.linear_cross_entropy(s["F"], s["X"], s["labels"], bias=s["bias"], ignore_index=_IGNORE)
        if not case["train"]:
            return loss, lse
        return (loss, lse) + lt.linear_cross_entropy_backward(s["F"], s["X"], s["labels"], lse, s["dloss"], bias=s["bias"],
                                                              ignore_index=_IGNORE)
    loss, lse = lt.linear_distill(s["F"], s["X"], s["top"], s["index"], bias=s["bias"], temperature=case["temperature"])
    if not case["train"]:
        return loss, lse
    return (loss, lse) + lt.linear_distill_backward(s["F"], s["X"], s["top"], s["index"], lse, s["dloss"], bias=s["bias"],
                                                    temperature=case["temperature"])


def work(case):
    """Each input once and each output once; products: one for the logits, three
    for the gradients, the logits among them again, since they are not kept."""
    size = _BYTES[case["dtype"]]
    if case["kind"] == "norm":
        n = case["c"] * case["h"] * case["w"] * case["b"]
        small = 4 * case["c"] * size + 8 * case["groups"] * case["b"]
        return {"bytes": float(size * n * (5 if case["train"] else 2) + small), "flops": float(n * (24 if case["train"] else 9))}
    kn, ci, t = case["kn"], case["ci"], case["t"]
    values = kn * ci + ci * t + (kn if case["bias"] else 0)
    tokens = 8 * t + (8 * t if case["kind"] == "loss" else (8 + size) * t * case["k"])
    if case["train"]:
        values += kn * ci + ci * t + kn
        tokens += 4 * t
    return {"bytes": float(size * values + tokens), "flops": (8.0 if case["train"] else 2.0) * kn * ci * t}


# ---------------------------------------------------------------------------
# the definition, in 64 bits
# ---------------------------------------------------------------------------
def _value(z, act):
    """The activation through the logistic and the complementary error function."""
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return z * torch.erfc(-z / math.sqrt(2.0)) / 2
    if act == "gelu_tanh":
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return torch.where(z > 0, 1.0, 0.0).double()
    if act == "gelu":
        return torch.erfc(-z / math.sqrt(2.0)) / 2 + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        gate = lambda v: 1 / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))     # noqa: E731
        return gate(z) + z * 2 * gate(z) * gate(-z) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z ** 2)
    return 1 / (1 + torch.exp(-z)) + z / ((1 + torch.exp(-z)) * (1 + torch.exp(z)))


def _exact_norm(s):
    case = s["case"]
    shape, g = (case["c"], case["h"], case["w"], case["b"]), case["groups"]
    x = s["x"].double().reshape(g, shape[0] // g, case["h"] * case["w"], case["b"])
    n = x.shape[1] * x.shape[2]
    mean = x.sum((1, 2), keepdim=True) / n
    var = ((x - mean) ** 2).sum((1, 2), keepdim=True) / n
    rstd = (var + _EPS) ** -0.5
    xhat = (x - mean) * rstd
    weight, bias = (s[k].double().reshape(g, -1, 1, 1) for k in ("weight", "bias"))
    z = xhat * weight + bias
    out = (_value(z, case["act"]).reshape(shape), mean.reshape(g, -1), rstd.reshape(g, -1))
    if not case["train"]:
        return out
    dz = s["dO"].double().reshape(x.shape) * _slope(z, case["act"])
    d = dz * weight
    # the derivative of (x - mean) / sqrt(var + eps) by every value of the group
    through_mean = d.sum((1, 2), keepdim=True) / n
    through_var = (d * xhat).sum((1, 2), keepdim=True) / n
    return out + ((rstd * (d - through_mean - xhat * through_var)).reshape(shape), (dz * xhat).sum((2, 3)).reshape(-1),
                  dz.sum((2, 3)).reshape(-1))


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(s)
    F, X, t = s["F"].double(), s["X"].double(), case["t"]
    z = torch.matmul(F, X)
    if s["bias"] is not None:
        z += s["bias"].double().unsqueeze(1)
    tokens = torch.arange(t, device="cuda")
    if case["kind"] == "loss":
        temperature, weight = 1.0, (s["labels"] != _IGNORE).double()
        entries = [(torch.where(s["labels"] < 0, 0, s["labels"]), torch.ones_like(weight))]
        entropy = torch.zeros_like(weight)
    else:
        temperature, weight = case["temperature"], torch.ones(t, dtype=torch.float64, device="cuda")
        log_q = torch.log_softmax(s["top"].double() / temperature, dim=0)
        entries = [(s["index"][i], torch.exp(log_q[i])) for i in range(case["k"])]
        entropy = -(torch.exp(log_q) * log_q).sum(0)
    z /= temperature
    lse = torch.logsumexp(z, dim=0)
    cross = sum(q * (lse - z[at, tokens]) for at, q in entries)
    loss = weight * temperature ** 2 * (cross - entropy)
    if not case["train"]:
        return loss, lse
    dz = z.sub_(lse).exp_()
    for at, q in entries:                       # one word a token each: no index twice
        dz[at, tokens] -= q
    dz *= s["dloss"].double() * weight * temperature
    return loss, lse, torch.matmul(F.t(), dz), torch.matmul(dz, X.t()), dz.sum(dim=1)
