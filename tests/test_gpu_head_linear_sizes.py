"""The first-order layer at sizes that one launch cannot take, 2^32 threads or 65535 rows of blocks; against
exact products."""
import pytest
import torch

import paper_2204_01701_amd as ql

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def _whole(*shape, seed=71):
    """Whole numbers of few bits: their short products are exact in any order."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-3, 4, shape, generator=g, device=DEV, dtype=torch.int8).to(BF)


def test_one_row_of_many_outputs():
    n = 2 ** 27 + 21
    x, w = _whole(2, 2), _whole(n, 2, seed=72)
    y = torch.empty(2, n, device=DEV, dtype=BF)
    ql.qhead_linear_fwd(x, w, None, None, y)
    for i in range(2):
        assert torch.equal(y[i], w[:, 0] * x[i, 0] + w[:, 1] * x[i, 1])


def test_many_rows_element_by_element(monkeypatch):
    monkeypatch.setenv("QHEAD_TILE", "1")
    m = 2 ** 30 + 5
    x, w = _whole(m, 1), torch.full((1, 1), 3.0, device=DEV, dtype=BF)
    y = torch.empty(m, 1, device=DEV, dtype=BF)
    ql.qhead_linear_fwd(x, w, None, None, y)
    assert torch.equal(y, x * 3)


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("m", [17, 0])
def test_gradients_of_long_rows(m, dtype):
    """Rows too long to be copied (2^31 / 256 bytes), in more than 65535 blocks of 64 columns."""
    k, n = 64 * 65537 + 7, 3
    x, w, dy = _whole(m, k).to(dtype), _whole(n, k, seed=73).to(dtype), _whole(m, n, seed=74).to(dtype)
    dx, dw, db = torch.empty(m, k, device=DEV, dtype=dtype), torch.empty(n, k, device=DEV, dtype=dtype), torch.empty(n, device=DEV)
    ql.qhead_linear_bwd(x, w, dy, None, dx, dw, db)
    assert torch.equal(dx, sum((dy[:, j:j + 1].float() * w[j].float() for j in range(n))).to(dtype))
    assert torch.equal(dw, sum((dy[i][:, None].float() * x[i].float() for i in range(m)), torch.zeros(n, k, device=DEV)).to(dtype))
    assert torch.equal(db, dy.float().sum(0))
