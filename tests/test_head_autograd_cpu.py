"""The autograd functions of the operators at the end of a network, as far as they are torch's
bookkeeping: run on the CPU with stand-ins for the library's calls that fill every output."""
import pytest
import torch

from paper_2204_01701_amd import autograd as ag


@pytest.fixture
def calls(monkeypatch):
    """The library's calls replaced; each call's tensors by name."""
    seen = []
    outputs = ("y", "z", "dx", "dw", "db", "logp", "entropy", "top_logp", "top_ids", "stats", "loss", "dlogits")
    names = {"qhead_linear_fwd": "x w b res y z", "qhead_linear_bwd": "x w dy z dx dw db",
             "qhead_logprobs_fwd": "logits target logp entropy lse top_logp top_ids stats",
             "qhead_logprobs_bwd": "logits target stats entropy g h dlogits",
             "qhead_distill_fwd": "logits t_ids t_logits labels loss stats",
             "qhead_distill_bwd": "logits t_ids t_logits labels stats g dlogits"}

    def stand_in(name):
        def call(*args, **kw):
            got = {**dict(zip(names[name].split(), args)), "call": name}
            for k in outputs:
                if got.get(k) is not None and not (name.endswith("_bwd") and k in ("z", "stats", "entropy")):
                    got[k].fill_(1)
            seen.append(got)
        return call

    monkeypatch.setattr(ag, "_same_device", lambda *tensors: None)  # (it asks for a GPU)
    for name in names:
        monkeypatch.setattr(ag, name, stand_in(name))
    return seen


def _linear(act, **needs):
    x, w, b, r = (torch.randn(s, requires_grad=needs.get(n, True)) for n, s in
                  (("x", (4, 5)), ("w", (3, 5)), ("b", (3,)), ("r", (4, 3))))
    return (x, w, b, r), ag.linear_act(x, w, b, r, act=act)


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("wrt", [0, 1, 2])
def test_a_second_derivative_of_the_layer_raises(calls, act, wrt):
    leaves, y = _linear(act)
    up = torch.randn_like(y).requires_grad_(True)
    g, = torch.autograd.grad(y, leaves[wrt], up, create_graph=True)
    with pytest.raises(RuntimeError, match="twice"):
        torch.autograd.grad(g.square().sum(), up)


@pytest.mark.parametrize("wrt", [0, 1])
def test_a_gradient_penalty_raises(calls, wrt):
    """The upstream gradient is a constant here; the gradient depends on the other factor, and on z."""
    for act in ("none", "gelu"):
        leaves, y = _linear(act)
        g, = torch.autograd.grad(y.sum(), leaves[wrt], create_graph=True)
        with pytest.raises(RuntimeError, match="twice"):
            torch.autograd.grad(g.square().sum(), leaves[1 - wrt], retain_graph=True, allow_unused=True)
        with pytest.raises(RuntimeError, match="twice"):
            (g.square().sum() + y.sum()).backward()


def test_what_does_not_depend_on_an_input_is_a_constant(calls):
    """dx = dy w with a frozen w, and db = sum dy: no second derivative is lost, none is refused."""
    (x, _, b, _), y = _linear("none", w=False)
    gx, gb = torch.autograd.grad(y.sum(), (x, b), create_graph=True)
    assert not gx.requires_grad and not gb.requires_grad
    (gx.sum() + gb.sum() + y.sum()).backward()


def test_the_residuals_gradient_stays_differentiable(calls):
    (_, _, _, r), y = _linear("silu")
    up = torch.randn_like(y).requires_grad_(True)
    g, = torch.autograd.grad(y, r, up, create_graph=True)
    again, = torch.autograd.grad(g.square().sum(), up)
    assert torch.equal(again, 2 * up)


@pytest.mark.parametrize("lead", [(4,), (2, 3)])
def test_second_derivatives_of_the_log_probabilities_and_the_loss_raise(calls, lead):
    z = torch.randn(*lead, 7, requires_grad=True)
    target = torch.zeros(lead, dtype=torch.int64)
    for out in (lambda: ag.token_logprobs(z, target)[0], lambda: ag.token_logprobs(z, target)[1],
                lambda: ag.distill_loss(z, None, None, target, alpha=0.0)):
        g, = torch.autograd.grad(out().sum(), z, create_graph=True)
        assert g.shape == z.shape
        with pytest.raises(RuntimeError, match="twice"):
            torch.autograd.grad(g.square().sum(), z, retain_graph=True, allow_unused=True)
        with pytest.raises(RuntimeError, match="twice"):
            g.square().sum().backward()


def test_first_derivatives_hold_no_graph(calls):
    leaves, y = _linear("silu")
    for g in torch.autograd.grad(y.sum(), leaves):
        assert not g.requires_grad
    z = torch.randn(4, 7, requires_grad=True)
    g, = torch.autograd.grad(ag.token_logprobs(z, torch.zeros(4, dtype=torch.int64))[0].sum(), z)
    assert not g.requires_grad


@pytest.mark.parametrize("off", [torch.no_grad, torch.inference_mode])
def test_serving_writes_nothing_for_a_backward(calls, off):
    """Parameters require gradients, the pass does not: no pre-activation and no statistics are asked for."""
    z, target = torch.randn(4, 7, requires_grad=True), torch.zeros(4, dtype=torch.int64)
    with off():
        y = _linear("gelu")[1]
        logp = ag.token_logprobs(z, target, top=2)[0]
        loss = ag.distill_loss(z, None, None, target, alpha=0.0)
    assert not (y.requires_grad or logp.requires_grad or loss.requires_grad)
    assert [c["call"] for c in calls] == ["qhead_linear_fwd", "qhead_logprobs_fwd", "qhead_distill_fwd"]
    assert calls[0]["z"] is None and calls[1]["stats"] is None and calls[2]["stats"] is None


def test_training_asks_for_them(calls):
    z, target = torch.randn(4, 7, requires_grad=True), torch.zeros(4, dtype=torch.int64)
    _linear("gelu"), ag.token_logprobs(z, target), ag.distill_loss(z, None, None, target, alpha=0.0)
    assert calls[0]["z"] is not None and calls[1]["stats"] is not None and calls[2]["stats"] is not None
    _linear("none")
    assert calls[3]["z"] is None


def test_functions_called_with_their_first_arguments_only(calls):
    x, w = torch.randn(4, 5, requires_grad=True), torch.randn(3, 5, requires_grad=True)
    z, target = torch.randn(4, 7, requires_grad=True), torch.zeros(4, dtype=torch.int64)
    ag.LinearActFunction.apply(x, w, None, None, "silu").sum().backward()
    ag.TokenLogprobsFunction.apply(z, target, 1.0, 0)[0].sum().backward()
    ag.DistillLossFunction.apply(z, None, None, target, 1.0, 0.5).sum().backward()
    assert x.grad is not None and w.grad is not None and z.grad is not None


@pytest.mark.parametrize("student", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("teacher", [torch.bfloat16, torch.float32, torch.float16])
def test_the_teachers_logits_lose_no_bits(calls, student, teacher):
    z = torch.randn(4, 7).to(student).requires_grad_(True)
    tz, ids = torch.randn(4, 3).to(teacher), torch.zeros(4, 3, dtype=torch.int64)
    ag.distill_loss(z, ids, tz).sum().backward()
    for c in calls:
        assert torch.equal(c["t_logits"].double(), tz.double())
        assert c["t_logits"].dtype in (student, torch.float32)


def test_a_float32_weights_gradient_is_asked_for_in_float32(calls):
    for xt, wt, want in ((torch.bfloat16, torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16, torch.bfloat16),
                         (torch.float32, torch.bfloat16, torch.float32), (torch.float32, torch.float32, torch.float32)):
        x, w = torch.randn(4, 5).to(xt), torch.randn(3, 5).to(wt).requires_grad_(True)
        ag.linear_act(x, w).sum().backward()
        assert calls[-1]["dw"].dtype is want and w.grad.dtype is wt
