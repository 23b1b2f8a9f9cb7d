"""The distillation's statistics at any float: a column range of a larger buffer, say."""
import pytest
import torch

import paper_2204_01701_amd as ql

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("offset", [1, 2, 3])
@pytest.mark.parametrize("rows,vocab", [(3, 20003), (300, 57), (2100, 700)])
def test_statistics_at_any_element(rows, vocab, offset):
    g = torch.Generator(device=DEV).manual_seed(91)
    z = torch.randn(rows, vocab, generator=g, device=DEV).bfloat16()
    label = torch.randint(vocab, (rows,), generator=g, device=DEV)
    ids, tz = torch.randint(vocab, (rows, 5), generator=g, device=DEV), torch.randn(rows, 5, generator=g, device=DEV)
    up, loss, dz = torch.randn(rows, generator=g, device=DEV), torch.empty(2, rows, device=DEV), torch.empty(2, *z.shape, device=DEV, dtype=z.dtype)
    plain, raw = torch.empty(rows, 4, device=DEV), torch.full((4 * rows + 8,), 77.0, device=DEV)
    stats = raw[offset:offset + 4 * rows].view(rows, 4)
    for i, st in enumerate((plain, stats)):
        ql.qhead_distill_fwd(z, ids, tz, label, loss[i], st, temperature=2.0, alpha=0.5)
        ql.qhead_distill_bwd(z, ids, tz, label, st, up, dz[i], temperature=2.0, alpha=0.5)
    assert torch.equal(loss[0], loss[1]) and torch.equal(dz[0], dz[1]) and torch.equal(plain, stats)
    assert bool((raw[:offset] == 77).all() and (raw[offset + 4 * rows:] == 77).all())
