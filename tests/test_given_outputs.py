"""Outputs that the caller gives: autograd sees that they were written, and one that
it records is refused."""

import pytest
import torch

import paper_2608_12573_amd as pk
from tests.gpu_util import note


def test_written_outputs_have_a_new_version():
    a, b = torch.zeros(3), torch.zeros(4)
    before = a._version, b._version
    pk._given(a, None, b)
    assert a._version > before[0] and b._version > before[1]
    leaf = torch.zeros(3, requires_grad=True)
    for t in (leaf, leaf * 2):
        with pytest.raises(pk.ProfkError, match="requires a gradient"):
            pk._given(a, t)
        with torch.no_grad():
            version = t._version
            pk._given(t)
            assert t._version > version


def _calls():
    """(name, call(**given outputs), the outputs) of every call that takes some."""
    g = torch.Generator().manual_seed(2)
    T, D, V, k = 6, 40, 70, 3
    f = dict(device="cuda")
    x, w = torch.randn((T, D), generator=g).bfloat16().cuda(), torch.randn((V, D), generator=g).bfloat16().cuda()
    logits, tokens = torch.randn((T, V), generator=g).cuda(), torch.randint(V, (T,), generator=g).cuda()
    _, m, r = pk.layer_norm(x)
    _, ent, lse, _, _ = pk.token_logprobs(logits, tokens)
    codes, scales = pk.mx4_quantize(w)
    one = torch.ones(T, **f)
    b_enc, w_dec, b_dec = torch.zeros(512, **f), torch.zeros((512, 64), dtype=torch.bfloat16, **f), torch.zeros(64, **f)
    h, enc = torch.randn((8, 64), generator=g).bfloat16().cuda(), torch.randn((512, 64), generator=g).bfloat16().cuda()
    bf = dict(dtype=torch.bfloat16, **f)
    flat = torch.randn(4096, generator=g).cuda()
    i64 = dict(dtype=torch.int64, **f)
    vals, idx = torch.zeros(5, **f), torch.zeros(5, **i64)
    return [
        ("layer_norm", lambda o: pk.layer_norm(x, out=o), pk.layer_norm_outputs(T, D)),
        ("layer_norm_grad", lambda o: pk.layer_norm_grad(x, x, None, m, r, out=o),
         (torch.empty((T, D), **bf), torch.empty(D, **f), None)),
        ("linear", lambda o: pk.linear(x, w, activation="relu", out=o[0], pre=o[1]),
         (torch.empty((T, V), **f), torch.empty((T, V), **f))),
        ("linear, pre alone", lambda o: pk.linear(x, w, activation="relu", pre=o[0]), (torch.empty((T, V), **f),)),
        ("linear_grad", lambda o: pk.linear_grad(logits, x, w, out=o),
         (torch.empty((T, D), **bf), torch.empty((V, D), **bf), torch.empty(V, **f))),
        ("adjust_logits", lambda o: pk.adjust_logits(logits, out=o[0]), (torch.empty((T, V), **f),)),
        ("adjust_logits_grad", lambda o: pk.adjust_logits_grad(logits, logits, out=o[0]), (torch.empty((T, V), **f),)),
        ("token_logprobs", lambda o: pk.token_logprobs(logits, tokens, k, out=o[:5], lse_low=o[5]),
         pk.token_logprobs_outputs(T, k) + (torch.empty(T, **f),)),
        ("token_logprobs_grad", lambda o: pk.token_logprobs_grad(logits, tokens, lse, ent, one, out=o[0]),
         (torch.empty((T, V), **f),)),
        ("mx4_dequantize", lambda o: pk.mx4_dequantize(codes, scales, D, out=o[0]), (torch.empty((V, D), **bf),)),
        ("mx4_matmul", lambda o: pk.mx4_matmul(codes, scales, codes, scales, D, out=o[0]), (torch.empty((V, V), **f),)),
        ("mx4_linear", lambda o: pk.mx4_linear(x, codes, scales, out=o[0]), (torch.empty((T, V), **f),)),
        ("mx4_quantize", lambda o: pk.mx4_quantize(w, out=o), pk.mx4_outputs(V, D)),
        ("topk", lambda o: pk.topk(flat, 5, out=o), (vals, idx)),
        ("topk_noalloc", lambda o: pk.topk_noalloc(flat, 5, out=o), (vals.clone(), idx.clone())),
        ("topk_rows", lambda o: pk.topk_rows(flat.view(4, 1024), 5, out=o), (torch.zeros(20, **f), torch.zeros(20, **i64))),
        ("batchtopk", lambda o: pk.batchtopk(flat.view(4, 1024), 5, out=o), (torch.zeros(20, **f), torch.zeros(20, **i64))),
        ("sae_encode_topk", lambda o: pk.sae_encode_topk(h, enc, b_enc, 4, out=o), (torch.zeros(32, **f), torch.zeros(32, **i64))),
        ("sae_encode_dense", lambda o: pk.sae_encode_dense(h, enc, b_enc, out=o[0]), (torch.zeros((8, 512), **f),)),
        ("sae_decode", lambda o: pk.sae_decode(vals, idx, w_dec, b_dec, 8, out=o[0]), (torch.zeros((8, 64), **f),)),
    ]


@pytest.mark.gpu
def test_every_call_shows_what_it_wrote():
    note("versions of given outputs")
    for name, call, outs in _calls():
        before = [None if o is None else o._version for o in outs]
        call(outs)
        for o, v in zip(outs, before):
            assert o is None or o._version > v, name
        for i, o in enumerate(outs):
            if o is None or not o.is_floating_point():
                continue
            leaf = o.clone().requires_grad_()
            given = outs[:i] + (leaf,) + outs[i + 1:]
            with pytest.raises(pk.ProfkError, match="requires a gradient"):
                call(given)
            with torch.no_grad():
                call(given)


@pytest.mark.gpu
def test_saved_rows_that_were_overwritten():
    note("a norm's rows overwritten by a product before its backward pass")
    g = torch.Generator().manual_seed(3)
    x = torch.randn((9, 64), generator=g).bfloat16().cuda()
    w, b = torch.ones(64, device="cuda", requires_grad=True), torch.zeros(64, device="cuda", requires_grad=True)
    w1 = torch.randn((64, 64), generator=g).bfloat16().cuda()
    y, _, _ = pk.layer_norm(x, w, b)
    pk.linear(y.detach(), w1, residual=x, out=x)
    with pytest.raises(RuntimeError, match="inplace"):
        y.float().sum().backward()
    # (and with nothing overwritten it passes)
    y, _, _ = pk.layer_norm(x, w, b)
    pk.linear(y.detach(), w1, residual=x, out=x.clone())
    y.float().sum().backward()
    assert torch.isfinite(w.grad).all()


@pytest.mark.gpu
def test_recorded_logits_are_not_adjusted_in_place():
    note("adjust_logits into recorded logits")
    g = torch.Generator().manual_seed(4)
    h = torch.randn((5, 64), generator=g).bfloat16().cuda()
    w = torch.randn((90, 64), generator=g).bfloat16().cuda().requires_grad_()
    tokens, at = torch.randint(90, (20,), generator=g).cuda(), torch.arange(6, device="cuda") * 4
    rep = torch.full((5,), 1.5, device="cuda")
    logits = pk.linear(h, w)
    with pytest.raises(pk.ProfkError, match="requires a gradient"):
        pk.adjust_logits(logits, tokens, at, repetition=rep, out=logits)
    # through a view of the same memory: what was saved of it is seen to have changed
    y = torch.exp(logits)
    with torch.no_grad():
        pk.adjust_logits(y, tokens, at, repetition=rep, out=y)
    with pytest.raises(RuntimeError, match="inplace"):
        y.sum().backward()
