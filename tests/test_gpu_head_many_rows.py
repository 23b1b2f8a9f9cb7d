"""More rows than one launch can take (2^32 threads): labels of every pixel of a batch, say.
Rows of few values, against float64 on the GPU, all of them."""
import pytest
import torch

import paper_2204_01701_amd as ql

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _case(rows, vocab, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = (torch.randn(rows, vocab, generator=g, device=DEV) * 2).to(dtype)
    return z, torch.randint(-1, vocab, (rows,), generator=g, device=DEV), torch.randn(rows, generator=g, device=DEV)


def _off(got, want, scale=1.0):
    """Largest error in units of the roundings: `scale` bounds the values, 64 float32 roundings of it and one to the type."""
    unit = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    off = (got.double() - want).abs_()
    return (off / (64 * 2.0 ** -24 * scale + unit * want.abs())).max().item()


@pytest.mark.parametrize("rows,vocab,dtype", [(2 ** 26 + 7, 2, torch.bfloat16), (2 ** 24 + 9, 3, torch.float32)])
def test_logprobs(rows, vocab, dtype):
    z, target, up = _case(rows, vocab, dtype, 61)
    logp, ent, lse, stats = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV)
    tl, ti = torch.empty(rows, 1, device=DEV), torch.empty(rows, 1, device=DEV, dtype=torch.int64)
    ql.qhead_logprobs_fwd(z, target, logp, ent, lse, tl, ti, stats)
    dz = torch.empty_like(z)
    ql.qhead_logprobs_bwd(z, target, stats, ent, up, up, dz)
    for part in torch.arange(rows, device=DEV).split(2 ** 24):  # (the whole at once in float64 would take the memory of all else)
        zs, t, u = z[part].double(), target[part], up[part].double()[:, None]
        full = torch.log_softmax(zs, 1)
        p = full.exp()
        picked = torch.where(t >= 0, full.gather(1, t.clamp_min(0)[:, None])[:, 0], 0.0)
        h = -(p * full).sum(1)
        best = torch.max(zs, 1)
        for got, want in ((logp, picked), (ent, h), (lse, torch.logsumexp(zs, 1)), (tl[:, 0], full.amax(1))):
            assert _off(got[part], want, 16.0) <= 1
        first = (zs == best[0][:, None]).int().argmax(1)
        assert torch.equal(ti[part, 0], first)
        one = torch.zeros_like(p).scatter_(1, t.clamp_min(0)[:, None], (t >= 0).double()[:, None])
        grad = u * (one - p * (t >= 0)[:, None]) - u * p * (full + h[:, None])
        assert _off(dz[part], grad, 64.0) <= 1


@pytest.mark.parametrize("rows,vocab,dtype", [(2 ** 26 + 7, 2, torch.bfloat16), (2 ** 24 + 9, 3, torch.float32)])
def test_cross_entropy(rows, vocab, dtype):
    z, label, up = _case(rows, vocab, dtype, 62)
    loss, dz, stats = torch.empty(rows, device=DEV), torch.empty_like(z), torch.empty(rows, 4, device=DEV)
    again, dz2 = torch.empty(rows, device=DEV), torch.empty_like(z)
    ql.qhead_distill_step(z, None, None, label, up, loss, dz, alpha=0.0)
    ql.qhead_distill_fwd(z, None, None, label, again, stats, alpha=0.0)
    ql.qhead_distill_bwd(z, None, None, label, stats, up, dz2, alpha=0.0)
    for part in torch.arange(rows, device=DEV).split(2 ** 24):
        zs, t, u = z[part].double(), label[part], up[part].double()[:, None]
        full = torch.log_softmax(zs, 1)
        given = (t >= 0).double()[:, None]
        one = torch.zeros_like(full).scatter_(1, t.clamp_min(0)[:, None], 1.0)
        want, grad = -(given * one * full).sum(1), u * given * (full.exp() - one)
        assert _off(loss[part], want, 16.0) <= 1 and _off(again[part], want, 16.0) <= 1
        assert _off(dz[part], grad, 16.0) <= 1 and _off(dz2[part], grad, 16.0) <= 1
