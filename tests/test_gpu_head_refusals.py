"""The binding refuses tensors that do not fit each other before anything is launched."""
import pytest
import torch

import paper_2204_01701_amd as ql
from paper_2204_01701_amd.autograd import distill_loss, linear_act, token_logprobs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def t(*shape, dtype=torch.float32):
    return torch.zeros(*shape, device=DEV, dtype=dtype)


def ids(*shape):
    return t(*shape, dtype=torch.int64)


BF = torch.bfloat16
CALLS = [
    lambda: ql.qhead_linear_fwd(t(4, 8), t(6, 9), None, None, t(4, 6)),
    lambda: ql.qhead_linear_fwd(t(4, 8), t(6, 8, dtype=BF), None, None, t(4, 6)),
    lambda: ql.qhead_linear_fwd(t(4, 8), t(6, 8), t(7), None, t(4, 6)),
    lambda: ql.qhead_linear_fwd(t(4, 8, dtype=BF), t(6, 8, dtype=BF), t(6, dtype=BF), None, t(4, 6, dtype=BF)),
    lambda: ql.qhead_linear_fwd(t(4, 8), t(6, 8), None, t(4, 5), t(4, 6)),
    lambda: ql.qhead_linear_fwd(t(4, 8), t(6, 8), None, t(1, 6).expand(4, 6), t(4, 6)),
    lambda: ql.qhead_linear_fwd(t(8, 4).t(), t(6, 8), None, None, t(4, 6)),
    lambda: ql.qhead_linear_fwd(t(4, 8), t(6, 8), None, None, t(4, 6), t(4, 12)[:, :6]),
    lambda: ql.qhead_linear_fwd(t(4, 8), t(6, 8), None, None, t(4, 6), act="tanh"),
    lambda: ql.qhead_linear_fwd(t(2, 4, 8), t(6, 8), None, None, t(4, 6)),
    lambda: ql.qhead_linear_fwd(t(4, 8, dtype=torch.float16), t(6, 8, dtype=torch.float16), None, None, t(4, 6)),
    lambda: ql.qhead_linear_fwd(t(4, 8), torch.zeros(6, 8), None, None, t(4, 6)),
    lambda: ql.qhead_linear_bwd(t(4, 8), t(6, 8), t(4, 7), dx=t(4, 8)),
    lambda: ql.qhead_linear_bwd(t(4, 8), t(6, 8), t(4, 6), dx=t(4, 9)),
    lambda: ql.qhead_linear_bwd(t(4, 8), t(6, 8), t(4, 6), dw=t(6, 8, dtype=BF)),
    lambda: ql.qhead_linear_bwd(t(4, 8), t(6, 8), t(4, 6), z=t(6, 4).t(), dx=t(4, 8)),
    lambda: ql.qhead_logprobs_fwd(t(4, 50), ids(5), t(4)),
    lambda: ql.qhead_logprobs_fwd(t(4, 50), t(4), t(4)),
    lambda: ql.qhead_logprobs_fwd(t(4, 50), ids(4), t(4, dtype=BF)),
    lambda: ql.qhead_logprobs_fwd(t(4, 50), ids(4), t(4), top_logp=t(4, 3)),
    lambda: ql.qhead_logprobs_fwd(t(4, 50), ids(4), t(4), top_logp=t(4, 3), top_ids=ids(4, 2)),
    lambda: ql.qhead_logprobs_fwd(t(4, 100)[:, ::2], ids(4), t(4)),
    lambda: ql.qhead_logprobs_bwd(t(4, 50), ids(4), t(4, 3), t(4), t(4), t(4), t(4, 50)),
    lambda: ql.qhead_logprobs_bwd(t(4, 50), ids(4), t(4, 2), t(4), t(4), t(4), t(4, 64)[:, :50]),
    lambda: ql.qhead_distill_fwd(t(4, 50), ids(4, 3), None, None, t(4)),
    lambda: ql.qhead_distill_fwd(t(4, 50), ids(4, 3), t(4, 3, dtype=BF), None, t(4)),
    lambda: ql.qhead_distill_fwd(t(4, 50), ids(3, 3), t(4, 3), None, t(4)),
    lambda: ql.qhead_distill_fwd(t(4, 50), ids(4, 6)[:, :3], t(4, 3), None, t(4)),
    lambda: ql.qhead_distill_step(t(4, 50), ids(4, 3), t(4, 3), None, t(5), t(4), t(4, 50)),
    lambda: linear_act(t(4, 8), t(6, 9)),
    lambda: linear_act(t(4, 8), t(6, 8), t(1)),
    lambda: linear_act(t(4, 8), t(6, 8), residual=t(6)),
    lambda: linear_act(t(4, 8), t(6, 8), act="swish"),
    lambda: linear_act(t(4, 8), t(6, 8), torch.zeros(6)),
    lambda: token_logprobs(t(4, 50), ids(50)),
    lambda: token_logprobs(t(4, 50), t(4)),
    lambda: distill_loss(t(4, 50), ids(3, 2), t(3, 2)),
    lambda: distill_loss(t(4, 50), ids(4, 2), t(4, 2), ids(3), alpha=0.5),
]
STATUS = [
    lambda: ql.qhead_logprobs_fwd(t(4, 5), ids(4), t(4), top_logp=t(4, 6), top_ids=ids(4, 6)),
    lambda: ql.qhead_logprobs_fwd(t(4, 50), ids(4), t(4), temperature=0.0),
    lambda: token_logprobs(t(4, 500), ids(4), top=129),
    lambda: distill_loss(t(4, 50), ids(4, 2), t(4, 2), alpha=1.5),
    lambda: ql.qhead_distill_fwd(t(4, 50), ids(4, 129), t(4, 129), None, t(4)),
    lambda: ql.qhead_linear_bwd(t(4, 8), t(6, 8), t(4, 6)),
    lambda: ql.qhead_linear_bwd(t(4, 8), t(6, 8), t(4, 6), dx=t(4, 8), act="gelu"),
    lambda: ql.qhead_linear_bwd(t(4, 8), t(6, 8), t(4, 6), z=t(4, 6), dx=t(4, 8), act="gelu", workspace=t(4)),
]


@pytest.mark.parametrize("i", range(len(CALLS)))
def test_wrong_tensors(i):
    with pytest.raises(ValueError):
        CALLS[i]()


@pytest.mark.parametrize("i", range(len(STATUS)))
def test_wrong_arguments(i):
    with pytest.raises(ql.QLError):
        STATUS[i]()


def test_raw_stream_needs_a_workspace():
    st = torch.cuda.Stream()
    big = t(4, 200000)
    with pytest.raises(ValueError):
        ql.qhead_logprobs_fwd(big, ids(4), t(4), stream=st.cuda_stream)
    need = ql.lib().qhead_logprobs_fwd_workspace_size(ql.ctypes.byref(ql.HeadRowsDesc(4, 200000, 200000, 0, ql.QL_F32, 1.0, 0.0)))
    logp = t(4)
    torch.cuda.synchronize()
    ql.qhead_logprobs_fwd(big, ids(4), logp, stream=st.cuda_stream, workspace=torch.empty(need, dtype=torch.uint8, device=DEV))
    st.synchronize()
    assert torch.allclose(logp, torch.full_like(logp, -12.206073))
