"""The distillation example: the operators together, as a program uses them."""
import pytest
import torch

from paper_2204_01701_amd import distill

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_student_learns_from_the_teacher(dtype):
    losses, before, after = distill.run(steps=60, dtype=dtype)
    assert all(v == v and abs(v) < 1e4 for v in losses)
    assert sum(losses[-5:]) < 0.5 * sum(losses[:5])
    assert after["logp"] > before["logp"] + 1.0
    assert after["accuracy"] > 0.5 and after["agreement"] > 0.5


def test_gradients_of_a_step_against_float64():
    """Every weight's gradient of one step, fp32, against the same network in float64 with torch's own operations."""
    torch.manual_seed(0)
    dev, dt = "cuda:0", torch.float32
    data = distill.Data(30, 24, 3, dev)
    teacher, student = distill.Teacher(data, dt), distill.Student(24, 40, 30, dt, dev, 4)
    x, label = data.batch(50, dt)
    label[::7] = -1
    ids, tz, _ = teacher.top(x, 6, label)
    loss = distill.distill_loss(student.logits(x), ids, tz, label, temperature=2.0, alpha=0.7)
    got = torch.autograd.grad(loss.mean(), student.weights)
    w = [v.detach().double().cpu().requires_grad_(True) for v in student.weights]
    xd = x.double().cpu()
    h = torch.relu((xd @ w[0].t() + w[3]) * (xd @ w[1].t() + w[4]) + xd @ w[2].t() + w[5])
    h = h + torch.nn.functional.silu(h @ w[6].t() + w[7])
    z = h @ w[8].t() + w[9]
    q = torch.softmax(tz.double().cpu() / 2, 1)
    kl = (q * (q.log() - torch.log_softmax(z / 2, 1).gather(1, ids.cpu()))).sum(1)
    ce = torch.nn.functional.cross_entropy(z, label.cpu(), reduction="none", ignore_index=-1)
    want = torch.autograd.grad((0.7 * 4 * kl + 0.3 * ce).mean(), w)
    for a, b in zip(got, want):
        # products of a few tens of terms through four layers: some 100 roundings of 2^-24
        assert (a.double().cpu() - b).norm() <= 1e-5 * b.norm()
