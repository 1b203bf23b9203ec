"""Forward-mode derivatives, which the calls do not have, are refused, not lost."""

import pytest
import torch
import torch.autograd.forward_ad as forward

import paper_2608_12573_amd as pk
from tests.gpu_util import note


def test_tangents_are_refused():
    x = torch.zeros(3)
    assert not pk._recorded(x, None) and pk._recorded(None, x.clone().requires_grad_())
    with torch.no_grad():
        assert not pk._recorded(x.clone().requires_grad_())
    with forward.dual_level():
        dual = forward.make_dual(x, torch.ones(3))
        assert not pk._recorded(x)
        for grad in (True, False):
            with torch.set_grad_enabled(grad), pytest.raises(pk.ProfkError, match="forward-mode"):
                pk._recorded(x, dual)
    assert not pk._recorded(x)


@pytest.mark.gpu
def test_every_differentiable_call():
    note("calls of dual tensors")
    g = torch.Generator().manual_seed(1)
    x, w = (torch.randn((n, 24), generator=g).bfloat16().cuda() for n in (5, 7))
    v = torch.ones(24, device="cuda")
    b, r, l = torch.ones(7, device="cuda"), torch.ones((5, 7), device="cuda"), torch.ones((5, 7), device="cuda")
    y = torch.zeros(5, dtype=torch.int64, device="cuda")
    calls = [(lambda x, v: pk.layer_norm(x, v), (x, v)), (lambda x, v: pk.layer_norm(x, None, v), (x, v)),
             (pk.linear, (x, w, b)), (lambda r: pk.linear(x, w, None, None, r), (r,)), (pk.adjust_logits, (l,)),
             (lambda l: pk.token_logprobs(l, y), (l,)),
             (lambda l: pk.adjust_logits(l, out=torch.empty_like(r)), (l,))]
    for call, inputs in calls:
        call(*inputs)
        for i, t in enumerate(inputs):
            with forward.dual_level():
                dual = forward.make_dual(t, torch.ones_like(t))
                call(*inputs)
                with pytest.raises(pk.ProfkError, match="forward-mode"):
                    call(*inputs[:i], dual, *inputs[i + 1:])
