"""Gradients written over the logits they are computed from: bit for bit what a separate output
receives, on rows long enough that all of a workgroup's waves, and several workgroups, hold parts
of them, with the targets spread over all of these parts."""
import pytest
import torch

import head_ref as ref
import paper_2204_01701_amd as ql

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float32]
type_ids = ["bf16", "fp32"]
# few rows (split over workgroups), one workgroup a row, many rows; whole and partial last vectors
SIZES = [(1, 131072), (7, 40003), (64, 9001), (1100, 4096), (1100, 8197), (5000, 1000)]


def _case(rows, vocab, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = (torch.randn(rows, vocab, generator=g, device=DEV) * 3).to(dtype)
    # rising targets reach every thread's vectors; the first and last elements are among them
    target = torch.linspace(0, vocab - 1, rows, device=DEV, dtype=torch.float64).round().long()
    if rows > 4:
        target[2] = -1
    up, h = (torch.randn(rows, generator=g, device=DEV) for _ in range(2))
    return z, target, up, h


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("rows,vocab", SIZES)
@pytest.mark.parametrize("with_h", [False, True])
def test_logprobs(rows, vocab, dtype, with_h):
    z, target, up, h = _case(rows, vocab, dtype, 31)
    if rows == 1:
        target[0] = 3 * vocab // 4 + 5  # a vector of the last wave
    logp, ent, stats = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV)
    ql.qhead_logprobs_fwd(z, target, logp, ent, stats=stats, temperature=1.3)
    apart = torch.empty_like(z)
    ql.qhead_logprobs_bwd(z, target, stats, ent, up, h if with_h else None, apart, temperature=1.3)
    over = z.clone()
    ql.qhead_logprobs_bwd(over, target, stats, ent, up, h if with_h else None, over, temperature=1.3)
    assert torch.equal(over, apart)
    at = torch.linspace(0, rows - 1, min(rows, 6), device=DEV).long()
    want, bound = ref.logprobs_grad(z[at].cpu(), target[at].cpu(), 1.3, up[at].cpu(), h[at].cpu() if with_h else None)
    ref.near(over[at], want, bound, dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=type_ids)
@pytest.mark.parametrize("rows,vocab", SIZES)
@pytest.mark.parametrize("t,alpha", [(2.0, 1.0), (2.0, 0.4), (1.0, 0.4)])
def test_distillation(rows, vocab, dtype, t, alpha):
    z, label, up, _ = _case(rows, vocab, dtype, 32)
    top = 64
    ids = (label.clamp_min(0)[:, None] + torch.arange(top, device=DEV) * (vocab // top + 1)) % vocab
    g = torch.Generator(device=DEV).manual_seed(33)
    tz = torch.randn(rows, top, generator=g, device=DEV).to(dtype)
    how = dict(temperature=t, alpha=alpha)
    loss, stats = torch.empty(rows, device=DEV), torch.empty(rows, 4, device=DEV)
    ql.qhead_distill_fwd(z, ids, tz, label, loss, stats, **how)
    apart, over = torch.empty_like(z), z.clone()
    ql.qhead_distill_bwd(z, ids, tz, label, stats, up, apart, **how)
    ql.qhead_distill_bwd(over, ids, tz, label, stats, up, over, **how)
    assert torch.equal(over, apart)
    over = z.clone()
    ql.qhead_distill_step(z, ids, tz, label, up, loss, apart, **how)
    ql.qhead_distill_step(over, ids, tz, label, up, loss, over, **how)
    assert torch.equal(over, apart)
