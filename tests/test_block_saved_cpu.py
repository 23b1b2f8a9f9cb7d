"""Saved tensors that a hook brings back in another order of memory, of another dtype or of another shape: what the backward's
calls are given holds the values that were saved, at the strides that the call states, or the backward refuses.  No GPU: the
library's calls are replaced by a reader of the memory behind their pointers."""
import ctypes
import math

import pytest
import torch

from paper_2204_01701_amd import autograd as ag

SIZES = {torch.float32: 4, torch.int8: 1, torch.uint8: 1}


def read(ptr, shape, strides=None, dtype=torch.float32):
    """The values at a pointer as a kernel that knows only shape and strides takes them."""
    if strides is None:
        strides = [math.prod(shape[i + 1:]) for i in range(len(shape))]
    n = sum((s - 1) * d for s, d in zip(shape, strides)) + 1
    raw = bytearray(ctypes.string_at(ptr, n * SIZES[dtype]))
    return torch.frombuffer(raw, dtype=dtype).as_strided(shape, strides).clone()


@pytest.fixture
def calls(monkeypatch):
    """What the library's calls are given: (name, descriptor, pointers), or, by name, what a reader makes of them at the call."""
    seen, readers = [], {}

    def launch(name, desc, ptrs, index, query=None):
        seen.append((name, readers[name](desc, ptrs) if name in readers else None))

    monkeypatch.setattr(ag, "_same_device", lambda *tensors: None)
    monkeypatch.setattr(ag, "_block_launch", launch)
    launch.seen, launch.readers = seen, readers
    return launch


def turned(t):
    """The same values, the last dimension outermost in memory."""
    dims = list(range(t.dim()))[::-1]
    return t.permute(dims).contiguous().permute(dims)


def spread(t):
    """The same values, every other element of memory."""
    wide = torch.empty(*t.shape, 2, dtype=t.dtype)
    wide[..., 0] = t
    return wide[..., 0]


ORDERS = [turned, spread]


def only(i, f):
    """A hook that changes the i-th saved tensor alone."""
    count = [0]

    def unpack(t):
        count[0] += 1
        return f(t) if count[0] == i + 1 else t
    return unpack


def leaf(*shape):
    return torch.randn(*shape, requires_grad=True)


# --- the gated layer -------------------------------------------------------------------

M, K, N = 6, 40, 36


def read_gated(desc, ptrs):
    assert (desc.m, desc.k, desc.n) == (M, K, N)
    x, wg, wu, dh, z, q, e = ptrs[:7]
    out = {"wg": read(wg, (N, K), (desc.ldw, 1)), "wu": read(wu, (N, K), (desc.ldw, 1)), "dh": read(dh, (M, N), (desc.ldh, 1))}
    if x is not None:
        out["x"] = read(x, (M, K), (desc.ldx, 1))
    if z is not None:
        out["z"] = read(z, (2, M, N))
    if q is not None:
        out["q"], out["e"] = read(q, (2, M, N), dtype=torch.int8), read(e, (2, M, 2), dtype=torch.uint8)
    return out


def gated(calls, unpack, checkpoint=None):
    """(what the backward read without the hook, with it)."""
    calls.readers["qblock_gated_bwd"] = read_gated
    torch.manual_seed(3)
    leaves, dh = [leaf(M, K), leaf(N, K), leaf(N, K)], torch.randn(M, N)
    filled = torch.randn(2, M, N), torch.randint(-9, 9, (2, M, N), dtype=torch.int8), torch.randint(1, 9, (2, M, 2), dtype=torch.uint8)

    def write(desc, ptrs):  # what the forward leaves for the backward
        for p, t in zip(ptrs[6:9], filled):
            if p is not None:
                ctypes.memmove(p, t.data_ptr(), t.numel() * t.element_size())
    calls.readers["qblock_gated_fwd"] = write
    for hook in (lambda t: t, unpack):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, hook):
            h = ag.gated_linear(*leaves, checkpoint=checkpoint)
        torch.autograd.grad(h, leaves, dh)
    plain, hooked = [got for name, got in calls.seen if name == "qblock_gated_bwd"]
    return plain, hooked


@pytest.mark.parametrize("f", ORDERS)
@pytest.mark.parametrize("i", range(4), ids=["x", "wg", "wu", "z"])
def test_gated_layer(calls, i, f):
    plain, hooked = gated(calls, only(i, f))
    assert sorted(plain) == ["dh", "wg", "wu", "x", "z"]
    for name, t in plain.items():
        assert torch.equal(hooked[name], t), name


@pytest.mark.parametrize("f", ORDERS)
@pytest.mark.parametrize("i", range(2, 6), ids=["wg", "wu", "q", "e"])
def test_gated_layer_from_its_checkpoint(calls, i, f):
    plain, hooked = gated(calls, only(i, f), "int8")
    assert sorted(plain) == ["dh", "e", "q", "wg", "wu", "x"]
    for name, t in plain.items():
        if name != "x":  # (unpacked by a call that is not made here)
            assert torch.equal(hooked[name], t), name


WRONG = [lambda t: t.double(), lambda t: t[..., :-1], lambda t: t.unsqueeze(0)]


@pytest.mark.parametrize("f", WRONG, ids=["dtype", "shape", "dimensions"])
@pytest.mark.parametrize("i", range(4), ids=["x", "wg", "wu", "z"])
def test_gated_layer_refuses(calls, i, f):
    with pytest.raises(ValueError, match="saved"):
        gated(calls, only(i, f))


@pytest.mark.parametrize("f", WRONG, ids=["dtype", "shape", "dimensions"])
@pytest.mark.parametrize("i", range(2, 6), ids=["wg", "wu", "q", "e"])
def test_gated_layer_refuses_checkpoints(calls, i, f):
    with pytest.raises(ValueError, match="saved"):
        gated(calls, only(i, f), "int8")


# --- group norm ------------------------------------------------------------------------

MAP, GROUPS = (2, 36, 3, 5), 4


def read_norm(desc, ptrs):
    n, c, h, w = MAP
    assert (desc.n, desc.hw, desc.c, desc.groups) == (n, h * w, c, GROUPS)
    dy, x, q, e, gamma, beta, mean, rstd = ptrs[:8]
    out = {"dy": read(dy, (n, h, w, c)), "gamma": read(gamma, (c,)), "beta": read(beta, (c,)), "mean": read(mean, (n, GROUPS)),
           "rstd": read(rstd, (n, GROUPS))}
    if x is not None:
        out["x"] = read(x, (n, h, w, c))
    if q is not None:
        out["q"], out["e"] = read(q, (n * h * w, c), dtype=torch.int8), read(e, (n * h * w, 2), dtype=torch.uint8)
    return out


def norm(calls, unpack, checkpoint=None):
    calls.readers["qblock_norm_bwd"] = read_norm
    n, c, h, w = MAP
    torch.manual_seed(4)
    leaves, dy = [leaf(*MAP), leaf(c), leaf(c)], torch.randn(MAP)
    stats = torch.randn(2, n, GROUPS)
    filled = (stats[0], stats[1], torch.randint(-9, 9, (n * h * w, c), dtype=torch.int8), torch.randint(1, 9, (n * h * w, 2), dtype=torch.uint8))

    def write(desc, ptrs):
        for p, t in zip(ptrs[4:8], filled):
            if p is not None:
                ctypes.memmove(p, t.data_ptr(), t.numel() * t.element_size())
    calls.readers["qblock_norm_fwd"] = write
    for hook in (lambda t: t, unpack):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, hook):
            y = ag.group_norm_act(leaves[0], GROUPS, leaves[1], leaves[2], checkpoint=checkpoint)
        torch.autograd.grad(y, leaves, dy)
    plain, hooked = [got for name, got in calls.seen if name == "qblock_norm_bwd"]
    return plain, hooked


KEPT = [(None, i) for i in range(4)] + [("int8", i) for i in range(5)]
KEPT_IDS = ["x", "gamma", "beta", "stats", "kept q", "kept e", "kept gamma", "kept beta", "kept stats"]


@pytest.mark.parametrize("f", ORDERS)
@pytest.mark.parametrize("checkpoint,i", KEPT, ids=KEPT_IDS)
def test_group_norm(calls, checkpoint, i, f):
    plain, hooked = norm(calls, only(i, f), checkpoint)
    assert sorted(plain) == sorted(["dy", "gamma", "beta", "mean", "rstd"] + (["q", "e"] if checkpoint else ["x"]))
    for name, t in plain.items():
        assert torch.equal(hooked[name], t), name


@pytest.mark.parametrize("f", WRONG, ids=["dtype", "shape", "dimensions"])
@pytest.mark.parametrize("checkpoint,i", KEPT, ids=KEPT_IDS)
def test_group_norm_refuses(calls, checkpoint, i, f):
    with pytest.raises(ValueError, match="saved"):
        norm(calls, only(i, f), checkpoint)


# --- what the layers keep of their inputs and maps in 8 bits ---------------------------------

@pytest.fixture
def layer(calls, monkeypatch):
    """The layers' own calls replaced as well; what the reads of the checkpoints are given: (q, e) by the shape of q."""
    for name in ("qhead_linear_fwd", "qhead_linear_bwd", "qlayer_linear_fwd", "qlayer_linear_bwd", "qlayer_conv2d_fwd", "qlayer_conv2d_bwd_data",
                 "qlayer_conv2d_bwd_weight"):
        monkeypatch.setattr(ag, name, lambda *args, **kw: None)

    def pack(desc, ptrs):
        g = torch.Generator().manual_seed(desc.rows * 1000 + desc.cols)
        for p, shape, dtype, lo in ((ptrs[1], (desc.rows, desc.cols), torch.int8, -9), (ptrs[2], (desc.rows, -(-desc.cols // 32)), torch.uint8, 1)):
            t = torch.randint(lo, 9, shape, dtype=dtype, generator=g)
            ctypes.memmove(p, t.data_ptr(), t.numel())

    def unpack(desc, ptrs):
        return read(ptrs[0], (desc.rows, desc.cols), dtype=torch.int8), read(ptrs[1], (desc.rows, -(-desc.cols // 32)), dtype=torch.uint8)
    calls.readers.update(qblock_pack8=pack, qblock_unpack8=unpack)
    return calls


def layers():
    """name: leaves, layer, the places of the checkpoints among what is saved."""
    ws = [leaf(36, 40) for _ in range(3)]
    cs = [leaf(36, 40, 3, 3) for _ in range(3)]
    return {"linear": ([leaf(6, 40), leaf(36, 40)], lambda x, w: ag.linear_act(x, w, act="silu", checkpoint="int8"), (0, 1, 3, 4)),
            "gated": ([leaf(6, 40), leaf(36, 40), leaf(36, 40)], lambda *a: ag.gated_linear(*a, checkpoint="int8"), (0, 1)),
            "quadratic": ([leaf(6, 40), *ws], lambda *a: ag.quad_linear(*a, checkpoint="int8"), (0, 1, 5, 6, 7, 8)),
            "convolution": ([leaf(2, 40, 4, 5), *cs], lambda *a: ag.quad_conv2d(*a, pad=1, checkpoint="int8"), (0, 1, 5, 6, 7, 8))}


def read_back(layer, which, unpack):
    """What the reads of the checkpoints were given without the hook, with it."""
    leaves, f, _ = layers()[which]
    every = []
    for hook in (lambda t: t, unpack):
        layer.seen.clear()
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, hook):
            y = f(*leaves)
        torch.autograd.grad(y, leaves, torch.randn(y.shape))
        every.append([got for name, got in layer.seen if name == "qblock_unpack8"])
    return every


KEEPS = [(which, i) for which, (_, _, kept) in layers().items() for i in range(len(kept))]


@pytest.mark.parametrize("f", ORDERS)
@pytest.mark.parametrize("which,i", KEEPS)
def test_checkpoints(layer, which, i, f):
    # (saved tensors that are None do not come by a hook: those of the layers above are all there but the biases)
    plain, hooked = read_back(layer, which, at_kept(i, f))
    assert len(plain) == len(hooked) == len([k for w, k in KEEPS if w == which]) // 2
    for (q, e), (hq, he) in zip(plain, hooked):
        assert torch.equal(q, hq) and torch.equal(e, he)


def at_kept(i, f):
    """A hook that changes the i-th of the checkpoints' tensors alone (int8 and uint8 ones, in the order in which they were saved)."""
    count = [0]

    def unpack(t):
        if t.dtype not in (torch.int8, torch.uint8):
            return t
        count[0] += 1
        return f(t) if count[0] == i + 1 else t
    return unpack


@pytest.mark.parametrize("f", WRONG, ids=["dtype", "shape", "dimensions"])
@pytest.mark.parametrize("which,i", KEEPS)
def test_checkpoints_refuse(layer, which, i, f):
    with pytest.raises(ValueError, match="saved"):
        read_back(layer, which, at_kept(i, f))


# --- the first-order layer's weight beside its checkpoints -----------------------------------

def linear(layer, unpack, act="none"):
    """(weight as the backward read it without the hook, with it)."""
    def read_linear(desc, ptrs):
        assert (desc.m, desc.k, desc.n) == (M, K, N)
        return read(ptrs[1], (N, K), (desc.ldw, 1))
    layer.readers["qhead_linear_bwd"] = read_linear
    leaves = [leaf(M, K), leaf(N, K)]
    for hook in (lambda t: t, unpack):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, hook):
            y = ag.linear_act(*leaves, act=act, checkpoint="int8")
        torch.autograd.grad(y, leaves, torch.randn(M, N))
    return [got for name, got in layer.seen if name == "qhead_linear_bwd"]


@pytest.mark.parametrize("f", ORDERS)
def test_first_order_layers_weight(layer, f):
    plain, hooked = linear(layer, only(2, f))
    assert torch.equal(plain, hooked)


@pytest.mark.parametrize("f", WRONG, ids=["dtype", "shape", "dimensions"])
def test_first_order_layers_weight_refuses(layer, f):
    with pytest.raises(ValueError, match="saved"):
        linear(layer, only(2, f))
