"""Sums over very many rows: the roundings of the parameters' gradients do not add up with the length of the batch.

Every term is the same value v = 1 + d.  Added up one by one in float32, the partial sums of the last 2^(p-1) of 2^p terms have a
last place of 2^(p-24), and with d a little below half of it each addition loses d: 2^p / 4 units of 2^-24 in all, where a sum of
sums over chains of L1 and L2 additions stays within L1 + L2."""
import pytest
import torch

import block_ref as ref
import paper_2204_01701_amd as ql

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def least_kept(p):
    """1 + d, which a float32 sum of 2^p of them rounds to 1 whenever it is added to the upper half of the sum."""
    return float(torch.tensor(1 + 0.98 * 2.0 ** (p - 25), dtype=torch.float32))


def test_norm_parameters():
    """2^20 rows of 4096: a workgroup takes 2048 batches of rows.  dgamma sums dz xh = rstd, dbeta sums dz = 1."""
    n, c, groups = 2**20, 4096, 32
    ones = torch.ones(n, 1, c, device=DEV, dtype=torch.bfloat16)  # (x and dy)
    v = least_kept(11)
    mean, rstd = torch.zeros(n, groups, device=DEV), torch.full((n, groups), v, device=DEV)
    dg, db = torch.empty(c, device=DEV), torch.empty(c, device=DEV)
    ql.qblock_norm_bwd(ones, ones, groups, None, None, mean, rstd, None, dg, db)
    assert bool((db == n).all())
    assert float((dg.double() - n * v).abs().max()) <= ref.DEPTH * ref.U32 * n * v


def test_gated_biases():
    """2^24 rows: dbu sums dh g = 1, dbg sums dh u = 1 + d.  128 rows of a thread, eight threads, the parts (64, and 32 of these sums)."""
    m, k, n = 2**24, 8, 4
    v = least_kept(14)
    z = torch.ones(2, m, n, device=DEV)
    z[1] = v
    dh, w = torch.ones(m, n, device=DEV), torch.zeros(n, k, device=DEV)
    dbg, dbu = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ql.qblock_gated_bwd(None, w, w, dh, z, dbg=dbg, dbu=dbu, act="none")
    assert bool((dbu == m).all())
    assert float((dbg.double() - m * v).abs().max()) <= (128 + 8 + 64 + 32 + 8) * ref.U32 * m * v
