"""A matrix of one column whose column stride is not 1: torch takes it for
contiguous, and so no copy changes its strides."""

import pytest
import torch

import paper_2608_12573_amd as pk
from tests.gpu_util import note


def test_strides_of_one_column():
    x = torch.zeros(1, 4).t()
    assert x.shape == (4, 1) and x.is_contiguous() and x.stride(1) != 1
    for call in (pk.layer_norm, pk.adjust_logits, lambda t: pk.topk_rows(t, 1), pk.mx4_quantize):
        with pytest.raises(pk.ProfkError, match="CUDA tensor"):
            call(x)
    with pytest.raises(pk.ProfkError, match="rows at least D apart"):
        pk.layer_norm(torch.zeros(1, 1).expand(4, 1))
    with pytest.raises(pk.ProfkError, match="unit column stride"):
        pk.layer_norm(torch.zeros(8, 4)[:, ::2])


@pytest.mark.gpu
def test_gradients_of_one_column():
    note("gradients of one column")
    g = torch.Generator().manual_seed(1)
    x, w = (torch.randn((n, 24), generator=g).bfloat16().cuda() for n in (5, 1))
    d = torch.randn((1, 5), generator=g).cuda()
    a, b = x.clone().requires_grad_(), w.clone().requires_grad_()
    torch.autograd.backward(pk.linear(a, b).t(), d)                     # (arrives as a column of stride 5)
    for got, want in zip((a.grad, b.grad), pk.linear_grad(d.reshape(5, 1), x, w)):
        assert torch.equal(got, want)
    for stride in ((1, 5), (3, 7)):
        y = torch.empty_strided((5, 1), stride, device="cuda").copy_(d.t())
        for call in (lambda t: pk.layer_norm(t)[0], pk.adjust_logits, lambda t: pk.topk_rows(t, 1)[0]):
            assert torch.equal(call(y), call(d.reshape(5, 1)))
