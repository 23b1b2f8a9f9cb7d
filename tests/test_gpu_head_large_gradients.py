"""Upstream gradients of any size, as loss scaling makes them, over masked logits: a masked entry
has probability 0 and its gradient is 0, not infinity times 0."""
import math

import pytest
import torch

import head_ref as ref
import paper_2204_01701_amd as ql

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab", [(2, 30011), (300, 57), (2100, 700)])
@pytest.mark.parametrize("size,t", [(1e9, 1.0), (1e6, 1e-3), (1e20, 1.0), (1e30, 2.0)])
def test_log_probabilities(rows, vocab, dtype, size, t):
    g = torch.Generator().manual_seed(81)
    z = (torch.randn(rows, vocab, generator=g) * 3 * min(t, 1.0)).to(dtype)
    z[torch.rand(rows, vocab, generator=g) < 0.4] = -math.inf
    z[::3, 1::2] = torch.finfo(dtype).min  # masked by the type's lowest value
    z[:, 0] = 1.0
    target = torch.zeros(rows, dtype=torch.int64)
    up, h = (size * torch.randn(rows, generator=g) for _ in range(2))
    zd, td, upd, hd = (v.to(DEV) for v in (z, target, up, h))
    logp, ent, stats = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV)
    ql.qhead_logprobs_fwd(zd, td, logp, ent, stats=stats, temperature=t)
    dz = torch.empty_like(zd)
    ql.qhead_logprobs_bwd(zd, td, stats, ent, upd, hd, dz, temperature=t)
    want, bound = ref.logprobs_grad(z, target, t, up, h)
    # (a probability below float32's smallest normal number is 0: size / t times 2^-126 and its logarithm)
    ref.near(dz, want, bound + 128 * 2.0 ** -126 * size / t, dtype)
    assert bool((dz.cpu()[z == -math.inf] == 0).all())
