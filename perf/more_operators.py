"""The operators of a block that is trained with its activations in 8 bits, as a program calls them.

Three operators, beside the quadratic layers and the end of a network:

* ``norm``: group normalisation of channels-last maps with an activation, y = act(gamma xh + beta)
  with xh = (x - mean) rstd over the pixels and channels of a group, and its gradients;
* ``gated``: the gated layer h = act(x Wg^T + bg) o (x Wu^T + bu), both projections, the activation
  and the product, and its gradients from the saved g and u;
* ``kept``: checkpoints of activations in 8 bits, blocks of 32 neighbours of a row with a power of two
  each: written and read back, and a first-order layer whose backward reads its input from one.

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
BLOCK = 32
EPS = 1e-5


def _norm(name, n, h, w, c, groups, act, dtype="bf16", way="fwd", int8=False):
    """x (n, h, w, c).  way "train": forward and backward through autograd.  int8: the backward reads x from a checkpoint."""
    d = dict(kind="norm", n=n, h=h, w=w, c=c, groups=groups, act=act, dtype=dtype, way=way, int8=int8)
    return dict(d, name=name) if name else d


def _gated(name, m, k, n, act, dtype="bf16", way="fwd", int8=False, bias=True, save=False, pad=0):
    """h (m, n) from x (m, k), whose rows lie `pad` elements apart.  save: the forward stores g and u; int8: the backward
    reads them from a checkpoint."""
    d = dict(kind="gated", m=m, k=k, n=n, act=act, dtype=dtype, way=way, int8=int8, bias=bias, save=save, pad=pad)
    return dict(d, name=name) if name else d


def _kept(name, rows, cols, dtype="bf16", way="trip", n=0):
    """way "trip": x (rows, cols) is packed and unpacked; "train": x w^T + b with n outputs, whose backward has x in 8 bits."""
    d = dict(kind="kept", rows=rows, cols=cols, dtype=dtype, way=way, n=n)
    return dict(d, name=name) if name else d


def listed():
    return [
        # A training step's norm in the last stage of a CIFAR ResNet: 256 maps of 8 x 8 x 64.
        _norm("norm_cifar_train", 256, 8, 8, 64, 8, "silu", dtype="fp32", way="train"),
        # The forward over the wide 32 x 32 maps of a CIFAR network at batch 128.
        _norm("norm_fwd", 128, 32, 32, 256, 32, "silu"),
        # Gradients on maps of 56 x 56 whose input was kept in 8 bits.
        _norm("norm_bwd_int8", 32, 56, 56, 256, 32, "gelu", way="bwd", int8=True),
        # Odd maps, groups of six channels, fp32, through autograd with the checkpoint.
        _norm("norm_ragged_fp32", 7, 31, 33, 174, 29, "silu", dtype="fp32", way="train", int8=True),
        # One token while serving: both projections' weights are read once.
        _gated("gated_one_token", 1, 4096, 8192, "silu"),
        # The forward of a training step (2048 -> 8192), g and u saved.
        _gated("gated_train_fwd", 8192, 2048, 8192, "silu", save=True),
        # Its gradients, from g and u in 8 bits.
        _gated("gated_bwd_int8", 4096, 2048, 8192, "gelu_tanh", way="bwd", int8=True),
        # fp32 at odd sizes through autograd, the rows of x cut out of a wider tensor.
        _gated("gated_ragged_fp32", 517, 1000, 1537, "gelu", dtype="fp32", way="train", pad=8),
        # The maps of a CIFAR stage, kept and read back, fp32.
        _kept("trip_cifar_fp32", 256 * 64, 64, dtype="fp32"),
        # Odd rows of a large activation.
        _kept("trip_large", 65537, 1000),
        # A training step of the large fully-connected layer with its input in 8 bits.
        _kept("kept_train", 8192, 4096, way="train", n=4096),
        # The same in fp32 at odd sizes.
        _kept("kept_ragged_fp32", 1021, 1537, dtype="fp32", way="train", n=1000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, q):
    """Half of the sizes are multiples of q, half of any kind."""
    v = _log(rng, lo, hi)
    return max(lo, v // q * q) if v >= q and rng.random() < 0.5 else v


def draw(rng):
    kind = rng.choice(["norm", "gated", "kept"])
    dtype = "bf16" if rng.random() < 0.65 else "fp32"
    most = 2.7e11 if dtype == "bf16" else 7e10
    if kind == "norm":
        # groups of 1 to 64 channels, or one group as a layer norm has it; maps from a single pixel to 112 x 112
        groups = rng.choice([1, 2, 4, 8, 16, 32, 32, rng.randint(3, 40)])
        c = groups * (rng.choice([2, 4, 8, 16, 32]) if rng.random() < 0.6 else _log(rng, 1, 64))
        case = _norm(None, _log(rng, 1, 512), _log(rng, 1, 112), _log(rng, 1, 112), c, groups, rng.choice(ACTS), dtype,
                     rng.choice(["fwd", "bwd", "train"]), rng.random() < 0.5)
        while case["n"] * case["h"] * case["w"] * c > 2.5e7:
            side = max(("n", "h", "w"), key=lambda s: case[s])
            case[side] = max(1, case[side] // 2)
        case["int8"] = case["int8"] and case["way"] != "fwd"
        if case["way"] != "fwd" and case["act"] == "relu":
            case["act"] = "silu"  # (the sign of a z next to 0 is a matter of the last bit: no two sides share its slope)
        return case
    if kind == "gated":
        way = rng.choice(["fwd", "fwd", "bwd"] if dtype == "bf16" else ["fwd", "bwd", "train"])
        case = _gated(None, _size(rng, 1, 8192, 16), _size(rng, 32, 4096, 64), _size(rng, 10, 8192, 64), rng.choice(ACTS), dtype,
                      way, way == "bwd" and rng.random() < 0.5, rng.random() < 0.7, way == "fwd" and rng.random() < 0.4,
                      rng.choice([0, 0, 8, 3]))
        if way == "train" and case["act"] == "relu":
            case["act"] = "gelu"  # (as above)
        while work(case)["flops"] > most:
            case["m"] = max(1, case["m"] // 2)
        return case
    if rng.random() < 0.5:
        case = _kept(None, _log(rng, 1, 131072), _size(rng, 1, 8192, 32), dtype)
        while case["rows"] * case["cols"] > 6e7:
            case["rows"] //= 2
        return case
    case = _kept(None, _size(rng, 1, 8192, 16), _size(rng, 32, 4096, 64), dtype, "train", _size(rng, 10, 4096, 64))
    while work(case)["flops"] > most:
        case["rows"] = max(1, case["rows"] // 2)
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


def _blocks(x):
    """(rows, blocks, 32) of a matrix, its rows filled up with zeros."""
    return torch.nn.functional.pad(x, (0, -x.shape[1] % BLOCK)).view(x.shape[0], -1, BLOCK)


def _power(e):
    """2^e for whole e from -126 to 127, from its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _pack(x):
    """The checkpoint of a matrix of finite values: q (rows, cols) int8 and the blocks' e + 127 (rows, blocks) uint8."""
    b = _blocks(x.float())
    top = b.abs().amax(2)
    part, power = torch.frexp(top)  # top = part 2^power, part in [1/2, 1)
    e = torch.where(part > 127 / 128, power - 6, power - 7).clamp_min(-126).masked_fill(top == 0, -126)
    q = torch.round(b * _power(-e)[..., None])
    return q.view(x.shape[0], -1)[:, : x.shape[1]].to(torch.int8).contiguous(), (e + 127).to(torch.uint8)


def _unpack(q, e):
    v = _blocks(q.float()) * _power(e.to(torch.int32) - 127)[..., None]
    return v.view(q.shape[0], -1)[:, : q.shape[1]]


def prepare(case, seed):
    dt, made = _dtype(case), _Inputs(seed)
    s = dict(case)
    if case["kind"] == "norm":
        n, h, w, c, g = (case[i] for i in ("n", "h", "w", "c", "groups"))
        # maps behind a layer with a bias: every channel has its own mean and width
        x = (made.normal(n, h, w, c) * (0.5 + made.normal(c).abs()) + made.normal(c)).to(dt)
        s.update(gamma=1 + made.normal(c, std=0.2), beta=made.normal(c, std=0.2), dy=made.normal(n, h, w, c, dtype=dt))
        if case["way"] == "train":
            # the layer's own view of a map: (n, c, h, w) in channels-last memory
            s.update(x=x.permute(0, 3, 1, 2).requires_grad_(True), dy=s["dy"].permute(0, 3, 1, 2))
            s["gamma"].requires_grad_(True)
            s["beta"].requires_grad_(True)
            return s
        stats = torch.empty(2, n, g, device=DEV)
        s.update(x=x, y=torch.empty_like(x), mean=stats[0], rstd=stats[1])
        if case["way"] == "bwd":
            xg = x.double().view(n, h * w, g, c // g)
            var, mean = torch.var_mean(xg, dim=(1, 3), correction=0)
            s.update(mean=mean.float(), rstd=torch.rsqrt(var + EPS).float(), dgamma=torch.empty(c, device=DEV), dbeta=torch.empty(c, device=DEV))
            if case["int8"]:
                s["q"], s["e"] = _pack(x.view(-1, c))
                s["x"] = None
        return s
    if case["kind"] == "gated":
        m, k, n = case["m"], case["k"], case["n"]
        std = 1 / math.sqrt(k)
        s.update(x=made.normal(m, k, dtype=dt, pad=case["pad"]), wg=made.normal(n, k, std=std, dtype=dt), wu=made.normal(n, k, std=std, dtype=dt),
                 bg=made.normal(n, std=0.1) if case["bias"] else None, bu=made.normal(n, std=0.1) if case["bias"] else None)
        if case["way"] == "fwd":
            s.update(out=torch.empty(m, n, device=DEV, dtype=dt), z=torch.empty(2, m, n, device=DEV, dtype=dt) if case["save"] else None)
            return s
        s["dh"] = made.normal(m, n, dtype=dt)
        if case["way"] == "train":
            for p in ("x", "wg", "wu", "bg", "bu"):
                if s[p] is not None:
                    s[p].requires_grad_(True)
            return s
        s.update(z=made.normal(2, m, n, dtype=dt), q=None, e=None, dx=torch.empty(m, k, device=DEV, dtype=dt),
                 dwg=torch.empty(n, k, device=DEV, dtype=dt), dwu=torch.empty(n, k, device=DEV, dtype=dt),
                 dbg=torch.empty(n, device=DEV) if case["bias"] else None, dbu=torch.empty(n, device=DEV) if case["bias"] else None)
        if case["int8"]:
            s["q"], s["e"] = (t.view(2, m, -1) for t in _pack(s["z"].view(2 * m, n)))
            s["z"] = None
        return s
    rows, cols, n = case["rows"], case["cols"], case["n"]
    # activations: most of them small, a few channels large, some rows nothing
    x = made.normal(rows, cols) * torch.exp(made.normal(cols))
    x = (x * (made.normal(rows, 1) > -2)).to(dt)
    if case["way"] == "trip":
        s.update(x=x, back=torch.empty_like(x), q=torch.empty(rows, cols, device=DEV, dtype=torch.int8),
                 e=torch.empty(rows, -(-cols // BLOCK), device=DEV, dtype=torch.uint8))
        return s
    s.update(x=x.requires_grad_(True), w=made.normal(n, cols, std=1 / math.sqrt(cols), dtype=dt).requires_grad_(True),
             b=made.normal(n, std=0.1).requires_grad_(True), dy=made.normal(rows, n, dtype=dt))
    return s


# --- one pass ----------------------------------------------------------------------

def run(s):
    return (_OWN if own else _PLAIN)[s["kind"]](s)


def _own_norm(s):
    import paper_2204_01701_amd as ql
    from paper_2204_01701_amd.autograd import group_norm_act

    if s["way"] == "train":
        y = group_norm_act(s["x"], s["groups"], s["gamma"], s["beta"], eps=EPS, act=s["act"], checkpoint="int8" if s["int8"] else None)
        return [y.detach(), *torch.autograd.grad(y, (s["x"], s["gamma"], s["beta"]), s["dy"])]
    if s["way"] == "fwd":
        ql.qblock_norm_fwd(s["x"], s["groups"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], act=s["act"], eps=EPS)
        return [s["y"], s["mean"], s["rstd"]]
    kept = dict(q=s["q"], e=s["e"]) if s["int8"] else {}
    ql.qblock_norm_bwd(s["dy"], s["x"], s["groups"], s["gamma"], s["beta"], s["mean"], s["rstd"], s["y"], s["dgamma"], s["dbeta"],
                       act=s["act"], **kept)
    return [s["y"], s["dgamma"], s["dbeta"]]


def _own_gated(s):
    import paper_2204_01701_amd as ql
    from paper_2204_01701_amd.autograd import gated_linear

    if s["way"] == "train":
        h = gated_linear(s["x"], s["wg"], s["wu"], s["bg"], s["bu"], act=s["act"])
        of = [s[p] for p in ("x", "wg", "wu", "bg", "bu") if s[p] is not None]
        return [h.detach(), *torch.autograd.grad(h, of, s["dh"])]
    if s["way"] == "fwd":
        ql.qblock_gated_fwd(s["x"], s["wg"], s["wu"], s["bg"], s["bu"], s["out"], s["z"], act=s["act"])
        return [s["out"], s["z"]]
    ql.qblock_gated_bwd(s["x"], s["wg"], s["wu"], s["dh"], s["z"], s["dx"], s["dwg"], s["dwu"], s["dbg"], s["dbu"], q=s["q"], e=s["e"],
                        act=s["act"])
    return [s["dx"], s["dwg"], s["dwu"], s["dbg"], s["dbu"]]


def _own_kept(s):
    import paper_2204_01701_amd as ql
    from paper_2204_01701_amd.autograd import linear_act

    if s["way"] == "trip":
        ql.qblock_pack8(s["x"], s["q"], s["e"])
        ql.qblock_unpack8(s["q"], s["e"], s["back"])
        return [s["back"], s["e"]]
    y = linear_act(s["x"], s["w"], s["b"], checkpoint="int8")
    return [y.detach(), *torch.autograd.grad(y, (s["x"], s["w"], s["b"]), s["dy"])]


def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _act_slope(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    sig = 1 / (1 + torch.exp(-z))
    return sig * (1 + z * (1 - sig))


def _plain_norm(s):
    n, h, w, c, g = (s[i] for i in ("n", "h", "w", "c", "groups"))
    dt, wide = _dtype(s), (n, h * w, g, c // g)
    gamma, beta = (s[p].detach().view(g, c // g) for p in ("gamma", "beta"))
    train = s["way"] == "train"
    x, dy = s["x"], s["dy"]
    if train:
        x, dy = (t.detach().permute(0, 2, 3, 1) for t in (x, dy))
    if s["way"] != "bwd":
        v = x.float().view(wide)
        mean = v.mean(dim=(1, 3), keepdim=True)
        v = v - mean
        rstd = torch.rsqrt((v * v).mean(dim=(1, 3), keepdim=True) + EPS)
        y = _act(v * rstd * gamma + beta, s["act"]).to(dt).view(n, h, w, c)
        if not train:
            return [y, mean.view(n, g), rstd.view(n, g)]
        y = y.permute(0, 3, 1, 2)
    else:
        mean, rstd = (s[p].view(n, 1, g, 1) for p in ("mean", "rstd"))
    if s["int8"]:
        x = _unpack(*(_pack(x.reshape(-1, c)) if train else (s["q"], s["e"])))
    xh = (x.float().view(wide) - mean) * rstd
    dz = dy.float().view(wide)
    if s["act"] != "none":
        dz = dz * _act_slope(xh * gamma + beta, s["act"])
    t = dz * gamma
    dx = rstd * (t - t.mean(dim=(1, 3), keepdim=True) - xh * (t * xh).mean(dim=(1, 3), keepdim=True))
    dx = dx.to(dt).view(n, h, w, c)
    rest = [(dz * xh).sum(dim=(0, 1)).view(c), dz.sum(dim=(0, 1)).view(c)]
    return [y, dx.permute(0, 3, 1, 2), *rest] if train else [dx, *rest]


def _plain_gated(s):
    dt, act = s["x"].dtype, s["act"]
    x, wg, wu = (s[p].detach().float() for p in ("x", "wg", "wu"))
    if s["way"] != "bwd":
        g, u = torch.mm(x, wg.t()), torch.mm(x, wu.t())
        if s["bg"] is not None:
            g, u = g + s["bg"].detach(), u + s["bu"].detach()
        h = (_act(g, act) * u).to(dt)
        if s["way"] == "fwd":
            return [h, torch.stack((g, u)).to(dt) if s["save"] else None]
    elif s["int8"]:
        m, n = s["m"], s["n"]
        g, u = _unpack(s["q"].view(2 * m, n), s["e"].view(2 * m, -1)).view(2, m, n)
    else:
        g, u = s["z"].float()
    dh = s["dh"].float()
    dg, du = dh * u * _act_slope(g, act), dh * _act(g, act)
    rest = [(torch.mm(dg, wg) + torch.mm(du, wu)).to(dt), torch.mm(dg.t(), x).to(dt), torch.mm(du.t(), x).to(dt)]
    if s["way"] == "train":
        return [h, *rest, *([dg.sum(0), du.sum(0)] if s["bg"] is not None else [])]
    return rest + ([dg.sum(0), du.sum(0)] if s["dbg"] is not None else [None, None])


def _plain_kept(s):
    x = s["x"].detach()
    q, e = _pack(x)
    back = _unpack(q, e)
    if s["way"] == "trip":
        return [back.to(x.dtype), e]
    w, dy = s["w"].detach().float(), s["dy"].float()
    y = torch.mm(x.float(), w.t()) + s["b"].detach()
    return [y.to(x.dtype), torch.mm(dy, w).to(x.dtype), torch.mm(dy.t(), back).to(x.dtype), dy.sum(0)]


_OWN = {"norm": _own_norm, "gated": _own_gated, "kept": _own_kept}
_PLAIN = {"norm": _plain_norm, "gated": _plain_gated, "kept": _plain_kept}


# --- what a pass cannot do without ---------------------------------------------------

def work(case):
    eb = 2 if case["dtype"] == "bf16" else 4
    kept = 1 + 1 / BLOCK  # bytes of a value in a checkpoint
    if case["kind"] == "norm":
        size, small = case["n"] * case["h"] * case["w"] * case["c"], 8 * case["n"] * case["groups"] + 16 * case["c"]
        fwd, bwd = 2 * eb * size, (2 * eb + (kept if case["int8"] else eb)) * size
        if case["way"] == "train":
            # (the checkpoint is written by the forward)
            return {"bytes": fwd + bwd + (kept * size if case["int8"] else 0) + 2 * small, "flops": 40.0 * size}
        return {"bytes": (fwd if case["way"] == "fwd" else bwd) + small, "flops": 16.0 * size}
    if case["kind"] == "gated":
        m, k, n = case["m"], case["k"], case["n"]
        fwd = eb * (m * k + 2 * n * k + m * n * (3 if case["save"] else 1)) + 8 * n
        bwd = eb * (2 * m * k + 4 * n * k + m * n) + 2 * m * n * (kept if case["int8"] else eb) + 8 * n
        if case["way"] == "train":
            return {"bytes": fwd + bwd + 2 * eb * m * n, "flops": 12.0 * m * k * n}
        return {"bytes": fwd if case["way"] == "fwd" else bwd, "flops": (4.0 if case["way"] == "fwd" else 8.0) * m * k * n}
    rows, cols, n = case["rows"], case["cols"], case["n"]
    if case["way"] == "trip":
        return {"bytes": 2 * (eb + kept) * rows * cols, "flops": 8.0 * rows * cols}
    m, k = rows, cols
    return {"bytes": eb * (2 * m * k + 3 * n * k + 2 * m * n) + 2 * kept * m * k + 8 * n, "flops": 6.0 * m * k * n}


# --- the definitions in 64 bits --------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "gated": _exact_gated, "kept": _exact_kept}[case["kind"]](s)


def _phi(act):
    f = torch.nn.functional
    return {"none": lambda u: u, "relu": torch.relu, "gelu": f.gelu, "silu": f.silu,
            "gelu_tanh": lambda u: f.gelu(u, approximate="tanh")}[act]


def _exact_kept_values(x):
    """What a checkpoint of x (rows, cols) stands for, in 64 bits: steps of the least power of two with 127 steps over the block."""
    b = _blocks(x.double())
    top = b.abs().amax(2, keepdim=True).clamp_min(2.0**-140)
    step = torch.exp2(torch.floor(torch.log2(top / 127)))
    step = torch.where(step * 127 < top, step * 2, step).clamp_min(2.0**-126)
    return ((b / step).round() * step).view(x.shape[0], -1)[:, : x.shape[1]]


def _exact_norm(s):
    n, h, w, c, g = (s[i] for i in ("n", "h", "w", "c", "groups"))
    gamma, beta = s["gamma"].detach().double().requires_grad_(True), s["beta"].detach().double().requires_grad_(True)
    if s["way"] == "bwd":
        x = (_unpack(s["q"], s["e"]).view(n, h, w, c) if s["int8"] else s["x"]).double().permute(0, 3, 1, 2)
        mean, rstd = s["mean"].double(), s["rstd"].double()
        dy = s["dy"].double().permute(0, 3, 1, 2)
    else:
        x = s["x"].detach().double() if s["way"] == "train" else s["x"].double().permute(0, 3, 1, 2)
        var, mean = torch.var_mean(x.reshape(n, g, -1), dim=2, correction=0)
        rstd = 1 / torch.sqrt(var + EPS)
        y = _phi(s["act"])(torch.nn.functional.group_norm(x, g, gamma, beta, EPS)).detach()
        if s["way"] == "fwd":
            return [y.permute(0, 2, 3, 1).contiguous(), mean, rstd]
        dy = s["dy"].double()
        if s["int8"]:
            x = _exact_kept_values(x.permute(0, 2, 3, 1).reshape(-1, c)).view(n, h, w, c).permute(0, 3, 1, 2)
    xh = ((x.reshape(n, g, -1) - mean[..., None]) * rstd[..., None]).view(n, c, h, w).requires_grad_(True)
    z = xh * gamma[:, None, None] + beta[:, None, None]
    dxh, dgamma, dbeta = torch.autograd.grad(_phi(s["act"])(z), (xh, gamma, beta), dy)
    v, u = dxh.reshape(n, g, -1), xh.detach().reshape(n, g, -1)
    dx = (v - v.mean(2, keepdim=True) - u * (u * v).mean(2, keepdim=True)) * rstd[..., None]
    dx = dx.view(n, c, h, w)
    return [y, dx, dgamma, dbeta] if s["way"] == "train" else [dx.permute(0, 2, 3, 1).contiguous(), dgamma, dbeta]


def _exact_gated(s):
    phi, x, wg, wu = _phi(s["act"]), *(s[p].detach().double() for p in ("x", "wg", "wu"))
    if s["way"] != "bwd":
        g, u = x @ wg.t(), x @ wu.t()
        if s["bg"] is not None:
            g, u = g + s["bg"].detach().double(), u + s["bu"].detach().double()
        if s["way"] == "fwd":
            return [phi(g) * u, torch.stack((g, u)) if s["save"] else None]
    elif s["int8"]:
        m, n = s["m"], s["n"]
        g, u = _unpack(s["q"].view(2 * m, n), s["e"].view(2 * m, -1)).double().view(2, m, n)
    else:
        g, u = s["z"].double()
    g, u = g.requires_grad_(True), u.requires_grad_(True)
    h = phi(g) * u
    dg, du = torch.autograd.grad(h, (g, u), s["dh"].double())
    rest = [dg @ wg + du @ wu, dg.t().contiguous() @ x, du.t().contiguous() @ x]
    if s["way"] == "train":
        return [h.detach(), *rest, *([dg.sum(0), du.sum(0)] if s["bg"] is not None else [])]
    return rest + ([dg.sum(0), du.sum(0)] if s["dbg"] is not None else [None, None])


def _exact_kept(s):
    x = s["x"].detach()
    back = _exact_kept_values(x)
    if s["way"] == "trip":
        return [back, None]
    x, w, dy = x.double(), s["w"].detach().double(), s["dy"].double()
    return [x @ w.t() + s["b"].detach().double(), dy @ w, dy.t().contiguous() @ back, dy.sum(0)]
