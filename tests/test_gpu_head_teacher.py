"""A teacher's logits in float32 beside a student's in bfloat16: the distillation's softmax of the
teacher is that of the values given, not of their bfloat16 roundings."""
import pytest
import torch

import head_ref as ref
import paper_2204_01701_amd as ql
from paper_2204_01701_amd.autograd import distill_loss, token_logprobs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _case(rows, vocab, top, seed=41):
    """Log probabilities around -10, where bfloat16 has steps of 1/16."""
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn(rows, vocab, generator=g) * 3).bfloat16()
    ids = torch.stack([torch.randperm(vocab, generator=g)[:top] for _ in range(rows)])
    tz = torch.randn(rows, top, generator=g) * 0.7 - 10.0
    ids[::5, -1] = -1
    tz[1::5, 0] = -float("inf")
    label = torch.randint(-1, vocab, (rows,), generator=g)
    return z, ids, tz, label, torch.randn(rows, generator=g)


# split rows, a wave a row, a workgroup a row, one that holds it in registers and one that reads it twice
@pytest.mark.parametrize("rows,vocab,top", [(3, 20003, 128), (2100, 100, 20), (40, 3001, 64), (300, 9001, 32), (260, 140003, 5)])
@pytest.mark.parametrize("t,alpha", [(1.0, 1.0), (2.0, 0.4)])
def test_against_float64(rows, vocab, top, t, alpha):
    z, ids, tz, label, up = _case(rows, vocab, top)
    at = torch.linspace(0, rows - 1, min(rows, 16)).long()
    want, grad, el, eg = ref.distill(z[at], ids[at], tz[at], label[at], t, alpha, up[at])
    zd, idsd, tzd, ld, upd = (v.to(DEV) for v in (z, ids, tz, label, up))
    how = dict(temperature=t, alpha=alpha)
    loss, stats, dz = torch.empty(rows, device=DEV), torch.empty(rows, 4, device=DEV), torch.empty_like(zd)
    ql.qhead_distill_fwd(zd, idsd, tzd, ld, loss, stats, **how)
    ref.near(loss[at.to(DEV)], want, el, torch.float32)
    ql.qhead_distill_bwd(zd, idsd, tzd, ld, stats, upd, dz, **how)
    ref.near(dz[at.to(DEV)], grad, eg, torch.bfloat16)
    ql.qhead_distill_step(zd, idsd, tzd, ld, upd, loss, dz, **how)
    ref.near(loss[at.to(DEV)], want, el, torch.float32)
    ref.near(dz[at.to(DEV)], grad, eg, torch.bfloat16)
    leaf = zd.clone().requires_grad_(True)
    mine = distill_loss(leaf, idsd, tzd, ld, **how)
    ref.near(mine[at.to(DEV)], want, el, torch.float32)
    ref.near(torch.autograd.grad(mine, leaf, upd)[0][at.to(DEV)], grad, eg, torch.bfloat16)


def test_from_the_alternatives_of_a_teacher():
    """token_logprobs' alternatives go to distill_loss as they are."""
    z, _, _, label, up = _case(50, 1000, 1)
    tl, ti = token_logprobs(z.to(DEV) * 0.5, label.to(DEV), top=20)[2:]
    assert tl.dtype == torch.float32
    want, _, el, _ = ref.distill(z, ti.cpu(), tl.cpu(), None, 1.0, 1.0, up)
    ref.near(distill_loss(z.to(DEV), ti, tl), want, el, torch.float32)


def test_a_bfloat16_teacher_beside_float32_logits_is_refused_by_the_binding():
    z, ids = torch.zeros(4, 50, device=DEV), torch.zeros(4, 3, dtype=torch.int64, device=DEV)
    with pytest.raises(ValueError):
        ql.qhead_distill_fwd(z, ids, torch.zeros(4, 3, device=DEV, dtype=torch.bfloat16), None, torch.zeros(4, device=DEV))
    with pytest.raises(ValueError):
        ql.qhead_distill_fwd(z.bfloat16(), ids, torch.zeros(4, 3, device=DEV, dtype=torch.float16), None, torch.zeros(4, device=DEV))
