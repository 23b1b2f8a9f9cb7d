"""The operators at the end of a network, as a program that trains or serves one calls them.

Three operators, from the last hidden layer to the loss or the answer:

* ``linear``: a first-order fully-connected layer with bias, activation and residual in the
  product's epilogue, y = act(x w^T + b) + r, and its gradients from the saved z = x w^T + b;
* ``logprobs``: the log probabilities of given tokens (or labels) under softmax(z / T), with the
  entropy and the most likely alternatives, and the gradient of the first two;
* ``distill``: the loss of a student's logits against a teacher's top logits, mixed with the
  label's cross entropy, and its gradient.

``run`` computes each in its plain form (elementary torch operations in 32 bits, rounded once at
the end), or, where ``own`` is true, through this repository's entry points.  ``exact`` computes
the same outputs from the definitions in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _linear(name, m, k, n, act, dtype="bf16", way="fwd", res=True, bias=True, pad=0):
    """y (m, n) from x (m, k) and w (n, k); the rows of x and r lie `pad` elements apart."""
    d = dict(kind="linear", m=m, k=k, n=n, act=act, dtype=dtype, way=way, res=res, bias=bias, pad=pad)
    return dict(d, name=name) if name else d


def _logprobs(name, rows, vocab, top, dtype="bf16", way="fwd", temperature=1.0, pad=0, masked=0.0):
    """`masked`: share of the logits that are -inf; `pad`: columns behind each row that are no logits."""
    d = dict(kind="logprobs", rows=rows, vocab=vocab, top=top, dtype=dtype, way=way, temperature=temperature, pad=pad,
             masked=masked)
    return dict(d, name=name) if name else d


def _distill(name, rows, vocab, top, dtype="bf16", way="step", temperature=2.0, alpha=1.0, pad=0):
    """way "step": loss and gradient in one call; "train": forward, then backward through autograd; "eval": the loss."""
    d = dict(kind="distill", rows=rows, vocab=vocab, top=top, dtype=dtype, way=way, temperature=temperature, alpha=alpha,
             pad=pad)
    return dict(d, name=name) if name else d


def listed():
    return [
        # One token through a 4096-wide layer while serving: the weights are read once.
        _linear("linear_one_token", 1, 4096, 4096, "silu"),
        # The forward of a training step on the large fully-connected layer of the benchmark.
        _linear("linear_train_fwd", 8192, 4096, 4096, "gelu"),
        # Gradients of an expanding layer (2048 -> 8192): input, weight and bias.
        _linear("linear_train_bwd", 4096, 2048, 8192, "gelu_tanh", way="bwd"),
        # fp32 at odd sizes, the rows of x cut out of a wider tensor.
        _linear("linear_ragged_fp32", 1021, 1000, 1537, "relu", dtype="fp32", pad=8),
        # The classifier of a CIFAR network: labels of a batch, the three best classes.
        _logprobs("score_cifar", 256, 10, 3, dtype="fp32"),
        # Four sequences being decoded: a large vocabulary, the sampled token and its alternatives.
        _logprobs("score_decode", 4, 131072, 20, temperature=0.8, masked=0.01),
        # A teacher's pass over a batch: the top logits that a student is trained on.
        _logprobs("score_teacher", 4096, 32768, 64),
        # Training on log probabilities with an entropy term: odd vocabulary in padded rows.
        _logprobs("train_logprobs_fp32", 1000, 50001, 0, dtype="fp32", way="train", pad=47),
        # Distilling a CIFAR classifier: all ten classes of the teacher and the label.
        _distill("distill_cifar", 256, 10, 10, dtype="fp32", temperature=4.0, alpha=0.7),
        # Distillation through autograd: odd rows and vocabulary, label mixed in.
        _distill("distill_train_ragged", 1023, 50001, 32, way="train", alpha=0.5),
        # The loss alone over an evaluation set, fp32.
        _distill("distill_eval_fp32", 2048, 21841, 50, dtype="fp32", way="eval", temperature=1.0, alpha=0.9),
        # The largest: a step over a large vocabulary.
        _distill("distill_step_large", 4096, 131072, 128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, q):
    """Half of the sizes are multiples of q, half of any kind."""
    v = _log(rng, lo, hi)
    return max(lo, v // q * q) if v >= q and rng.random() < 0.5 else v


def draw(rng):
    kind = rng.choice(["linear", "logprobs", "distill"])
    dtype = "bf16" if rng.random() < 0.65 else "fp32"
    if kind == "linear":
        way = rng.choice(["fwd", "bwd"])
        case = _linear(None, _size(rng, 1, 8192, 16), _size(rng, 32, 4096, 64), _size(rng, 10, 8192, 64), rng.choice(ACTS),
                       dtype, way, rng.random() < 0.5, rng.random() < 0.8, rng.choice([0, 0, 8, 3]))
        while work(case)["flops"] > (2.7e11 if dtype == "bf16" else 7e10):
            case["m"] = max(1, case["m"] // 2)
        return case
    vocab, pad = _size(rng, 10, 131072, 64), rng.choice([0, 0, 15, 64])
    top = min(vocab, rng.choice([0, 1, 5, 20, 64, 128] if kind == "logprobs" else [1, 8, 10, 32, 64, 128]))
    temperature = rng.choice([1.0, 0.7, 2.0, 4.0])
    if kind == "logprobs":
        way = rng.choice(["fwd", "fwd", "train"])
        case = _logprobs(None, _size(rng, 1, 8192, 16), vocab, top, dtype, way, temperature, pad, rng.choice([0.0, 0.02, 0.5]))
    else:
        case = _distill(None, _size(rng, 1, 8192, 16), vocab, top, dtype, rng.choice(["step", "train", "eval"]), temperature,
                        rng.choice([1.0, 0.5, 0.9]), pad)
    while case["rows"] * vocab > 1.4e8:
        case["rows"] //= 2
    return case


# --- inputs ----------------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


class _Inputs:
    """Seeded tensors on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV).manual_seed(int(seed))

    def normal(self, *shape, std=1.0, dtype=torch.float32, pad=0):
        t = torch.randn(*shape[:-1], shape[-1] + pad, generator=self.g, device=DEV) * std
        return t.to(dtype)[..., : shape[-1]]

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device=DEV)

    def whole(self, n, *shape):
        return torch.randint(0, n, shape, generator=self.g, device=DEV)


def prepare(case, seed):
    dt, made = _dtype(case), _Inputs(seed)
    s = dict(case)
    if case["kind"] == "linear":
        m, k, n, pad = case["m"], case["k"], case["n"], case["pad"]
        s.update(x=made.normal(m, k, dtype=dt, pad=pad), w=made.normal(n, k, std=1 / math.sqrt(k), dtype=dt),
                 b=made.normal(n, std=0.1) if case["bias"] else None)
        if case["way"] == "fwd":
            # y: where the layer's output goes
            s.update(r=made.normal(m, n, dtype=dt, pad=pad) if case["res"] else None, y=torch.empty(m, n, device=DEV, dtype=dt))
        else:
            # z: the pre-activation that the forward saved; the buffers that the gradients go to
            s.update(z=made.normal(m, n, dtype=dt), dy=made.normal(m, n, dtype=dt), dx=torch.empty(m, k, device=DEV, dtype=dt),
                     dw=torch.empty(n, k, device=DEV, dtype=dt), db=torch.empty(n, device=DEV) if case["bias"] else None)
        return s
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    # a model's logits: a bell around zero with a few tokens well above the rest
    z = made.normal(rows, vocab, std=2.5, pad=case["pad"])
    likely = made.whole(vocab, rows, min(8, vocab))
    z.scatter_add_(1, likely, 6.0 + 3.0 * made.normal(rows, likely.shape[1]))
    target = torch.where(made.uniform(rows) < 0.6, likely[:, 0], made.whole(vocab, rows))
    target = torch.where(made.uniform(rows) < 0.05, torch.full_like(target, -100), target)  # rows without a target
    if case["kind"] == "logprobs":
        if case["masked"]:
            hide = made.uniform(rows, vocab) < case["masked"]
            hide.scatter_(1, likely[:, :1], False)
            z.masked_fill_(hide, -math.inf)
        s.update(z=z.to(dt), target=target)
        if case["way"] == "train":
            s.update(g_logp=made.normal(rows, std=1 / rows), g_entropy=made.normal(rows, std=0.01 / rows))
            s["z"].requires_grad_(True)
        else:
            f = torch.empty(3, rows, device=DEV)
            s.update(logp=f[0], entropy=f[1], lse=f[2], top_logp=torch.empty(rows, top, device=DEV),
                     top_ids=torch.empty(rows, top, device=DEV, dtype=torch.int64))
        return s
    # the teacher agrees with the student in part; its last places of some rows are empty
    t = z * 0.8
    t += made.normal(rows, vocab, std=1.5)
    t_logits, t_ids = torch.topk(t, top, dim=1)
    del t
    empty = made.uniform(rows, 1) * 10 < torch.arange(top, device=DEV) / top - 0.7
    t_ids = t_ids.masked_fill(empty, -1)
    s.update(z=z.to(dt), t_ids=t_ids, t_logits=t_logits.to(dt), label=target if case["alpha"] < 1 else None,
             weight=(target >= 0).float() / rows, loss=torch.empty(rows, device=DEV))
    if case["way"] == "train":
        s["z"].requires_grad_(True)
    elif case["way"] == "step":
        s["dz"] = torch.empty(rows, vocab, device=DEV, dtype=dt)
    return s


# --- one pass ----------------------------------------------------------------------

def run(s):
    return (_OWN if own else _PLAIN)[s["kind"]](s)


def _own_linear(s):
    import paper_2204_01701_amd as ql

    if s["way"] == "fwd":
        ql.qhead_linear_fwd(s["x"], s["w"], s["b"], s["r"], s["y"], act=s["act"])
        return s["y"]
    ql.qhead_linear_bwd(s["x"], s["w"], s["dy"], s["z"], s["dx"], s["dw"], s["db"], act=s["act"])
    return [s["dx"], s["dw"], s["db"]]


def _own_logprobs(s):
    import paper_2204_01701_amd as ql
    from paper_2204_01701_amd.autograd import token_logprobs

    if s["way"] == "train":
        logp, entropy = token_logprobs(s["z"], s["target"], temperature=s["temperature"])
        dz, = torch.autograd.grad((logp, entropy), s["z"], (s["g_logp"], s["g_entropy"]))
        return [logp.detach(), entropy.detach(), dz]
    ql.qhead_logprobs_fwd(s["z"], s["target"], s["logp"], s["entropy"], s["lse"], s["top_logp"], s["top_ids"],
                          temperature=s["temperature"])
    return [s["logp"], s["entropy"], s["lse"], s["top_logp"], s["top_ids"]]


def _own_distill(s):
    import paper_2204_01701_amd as ql
    from paper_2204_01701_amd.autograd import distill_loss

    how = dict(temperature=s["temperature"], alpha=s["alpha"])
    if s["way"] == "train":
        loss = distill_loss(s["z"], s["t_ids"], s["t_logits"], s["label"], **how)
        dz, = torch.autograd.grad(loss, s["z"], s["weight"])
        return [loss.detach(), dz]
    if s["way"] == "eval":
        ql.qhead_distill_fwd(s["z"], s["t_ids"], s["t_logits"], s["label"], s["loss"], **how)
        return s["loss"]
    ql.qhead_distill_step(s["z"], s["t_ids"], s["t_logits"], s["label"], s["weight"], s["loss"], s["dz"], **how)
    return [s["loss"], s["dz"]]


def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    sig = 1 / (1 + torch.exp(-z))
    return sig * (1 + z * (1 - sig))


def _plain_linear(s):
    dt, x, w = s["x"].dtype, s["x"].float(), s["w"].float()
    if s["way"] == "fwd":
        z = torch.mm(x, w.t())
        if s["b"] is not None:
            z = z + s["b"]
        y = _act(z, s["act"])
        return (y + s["r"].float() if s["r"] is not None else y).to(dt)
    dz = s["dy"].float()
    if s["act"] != "none":
        dz = dz * _act_slope(s["z"].float(), s["act"])
    return [torch.mm(dz, w).to(dt), torch.mm(dz.t(), x).to(dt), dz.sum(0) if s["db"] is not None else None]


def _plain_log_softmax(z):
    """log softmax, its exponential and the log of the sum of exponentials, of rows with one finite entry at least."""
    top = z.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
    logp = z - lse
    return logp, torch.exp(logp), lse[:, 0]


def _plain_logprobs(s):
    z = s["z"].detach()
    logp, p, lse = _plain_log_softmax(z.float() / s["temperature"])
    plogp = torch.where(p > 0, p * logp, 0.0)
    entropy = -plogp.sum(1)
    target, given = s["target"], s["target"] >= 0
    at = target.clamp_min(0)[:, None]
    picked = torch.where(given, logp.gather(1, at)[:, 0], 0.0)
    if s["way"] == "train":
        g = torch.where(given, s["g_logp"], 0.0)
        dz = -g[:, None] * p - s["g_entropy"][:, None] * (plogp + p * entropy[:, None])
        dz.scatter_add_(1, at, g[:, None])
        return [picked, entropy, (dz / s["temperature"]).to(z.dtype)]
    order = torch.sort(z.float(), dim=1, descending=True, stable=True)[1][:, : s["top"]]
    return [picked, entropy, lse, logp.gather(1, order), order]


def _plain_distill(s):
    z, ids, label, temp, alpha = s["z"].detach(), s["t_ids"], s["label"], s["temperature"], s["alpha"]
    rows, step = z.shape[0], s["way"] != "eval"
    logp, p, _ = _plain_log_softmax(z.float() / temp)
    t = torch.where(ids >= 0, s["t_logits"].float() / temp, -math.inf)
    q = torch.exp(t - t.amax(1, keepdim=True))
    q = q / q.sum(1, keepdim=True)
    at = ids.clamp_min(0)
    loss = alpha * temp * temp * torch.where(q > 0, q * (torch.log(q) - logp.gather(1, at)), 0.0).sum(1)
    if step:
        dz = (alpha * temp) * p.scatter_add_(1, at, -q)
    if label is not None:
        given, at = label >= 0, label.clamp_min(0)[:, None]
        logp, p, _ = _plain_log_softmax(z.float())
        loss = loss - (1 - alpha) * torch.where(given, logp.gather(1, at)[:, 0], 0.0)
        if step:
            one = torch.full((rows, 1), -1.0, device=z.device)
            dz += (1 - alpha) * torch.where(given[:, None], p.scatter_add_(1, at, one), 0.0)
    return [loss, (dz * s["weight"][:, None]).to(z.dtype)] if step else loss


_OWN = {"linear": _own_linear, "logprobs": _own_logprobs, "distill": _own_distill}
_PLAIN = {"linear": _plain_linear, "logprobs": _plain_logprobs, "distill": _plain_distill}


# --- what a pass cannot do without ---------------------------------------------------

def work(case):
    eb = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        if case["way"] == "fwd":
            return {"bytes": eb * (m * k + n * k + m * n * (2 if case["res"] else 1)) + 4 * n, "flops": 2.0 * m * k * n}
        return {"bytes": eb * (2 * m * k + 2 * n * k + 2 * m * n) + 4 * n, "flops": 4.0 * m * k * n}
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    grad = case["way"] in ("train", "step")
    # the logits once, their gradient once, what is small per row; a dozen operations an element
    small = rows * (24 + 12 * top) if case["kind"] == "logprobs" else rows * (16 + (8 + eb) * top)
    return {"bytes": eb * rows * vocab * (2 if grad else 1) + small, "flops": 12.0 * rows * vocab}


# --- the definitions in 64 bits --------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        return {"linear": _exact_linear, "logprobs": _exact_logprobs, "distill": _exact_distill}[case["kind"]](s)


def _exact_linear(s):
    x, w = s["x"].double(), s["w"].double()
    phi = {"none": lambda u: u, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
           "gelu_tanh": lambda u: torch.nn.functional.gelu(u, approximate="tanh")}[s["act"]]
    if s["way"] == "fwd":
        z = x @ w.t()
        y = phi(z if s["b"] is None else z + s["b"].double())
        return y if s["r"] is None else y + s["r"].double()
    with torch.enable_grad():
        z = s["z"].double().requires_grad_(True)
        dz, = torch.autograd.grad(phi(z), z, s["dy"].double())
    return [dz @ w, dz.t().contiguous() @ x, None if s["db"] is None else dz.sum(0)]


def _exact_logprobs(s):
    z, target = s["z"].detach().double(), s["target"]
    rows = torch.arange(z.shape[0], device=z.device)
    with torch.enable_grad():
        z.requires_grad_(True)
        logp = torch.log_softmax(z / s["temperature"], 1)
        picked = torch.where(target >= 0, logp[rows, target.clamp_min(0)], 0.0)
        finite = logp.masked_fill(torch.isinf(logp), 0.0)
        entropy = -(torch.softmax(z / s["temperature"], 1) * finite).sum(1)
        if s["way"] == "train":
            dz, = torch.autograd.grad((picked, entropy), z, (s["g_logp"].double(), s["g_entropy"].double()))
            return [picked.detach(), entropy.detach(), dz]
    logp, lse = logp.detach(), torch.logsumexp(z.detach() / s["temperature"], 1)
    return [picked.detach(), entropy.detach(), lse, torch.topk(logp, s["top"], dim=1)[0], None]


def _exact_distill(s):
    z, ids, label, temp, alpha = s["z"].detach().double(), s["t_ids"], s["label"], s["temperature"], s["alpha"]
    with torch.enable_grad():
        z.requires_grad_(True)
        t = s["t_logits"].double().masked_fill(ids < 0, -math.inf)
        q = torch.softmax(t / temp, 1)
        kl = torch.special.xlogy(q, q) - q * torch.log_softmax(z / temp, 1).gather(1, ids.clamp_min(0))
        loss = alpha * temp**2 * kl.sum(1)
        if label is not None:
            loss = loss + (1 - alpha) * torch.nn.functional.cross_entropy(z, label, reduction="none", ignore_index=-100)
        if s["way"] == "eval":
            return loss.detach()
        dz, = torch.autograd.grad(loss, z, s["weight"].double())
    return [loss.detach(), dz]
