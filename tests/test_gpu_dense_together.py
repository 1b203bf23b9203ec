"""layer_norm, linear and adjust_logits as they are used together: a chain with
its gradients, in captured graphs, on other streams, and before the selections
and log probabilities that follow them."""

import os
import sys

import numpy as np
import pytest

import paper_2608_12573_amd as pk
from gpu_util import note, torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def _data(T, D, V, seed):
    t = torch()
    g = t.Generator().manual_seed(seed)
    n = t.randint(0, 30, (T,), generator=g)
    at = t.zeros(T + 1, dtype=t.int64)
    at[1:] = n.cumsum(0)
    d = dict(x=t.randn((T, D), generator=g).bfloat16(), w=1 + 0.1 * t.randn(D, generator=g), b=0.1 * t.randn(D, generator=g),
             w1=(t.randn((D, D), generator=g) / D ** 0.5).bfloat16(), c1=0.1 * t.randn(D, generator=g),
             w2=(t.randn((V, D), generator=g) / D ** 0.5).bfloat16(), y=t.randint(V, (T,), generator=g),
             tokens=t.randint(V, (int(at[-1]),), generator=g), offsets=at, rep=1 + t.rand(T, generator=g),
             allowed=t.randint(-2 ** 31, 2 ** 31, (2, -(-V // 32)), generator=g).to(t.int32),
             mask=t.randint(-1, 2, (T,), generator=g))
    return {k: v.cuda() for k, v in d.items()}


def _by_hand(d, g):
    """The chain's output and the gradients of x, w, b, w1, c1 and w2, call by
    call; g: the gradient of the log probabilities."""
    t = torch()
    y, m, r = pk.layer_norm(d["x"], d["w"], d["b"])
    z = t.empty_like(d["x"])
    h = pk.linear(y, d["w1"], d["c1"], "gelu", d["x"], dtype=t.bfloat16, pre=z)
    l0 = pk.linear(h, d["w2"])
    kw = dict(tokens=d["tokens"], offsets=d["offsets"], repetition=d["rep"], allowed=d["allowed"], mask=d["mask"])
    l1 = pk.adjust_logits(l0, **kw)
    low = t.empty(len(g), device="cuda")
    lp, ent, lse, _, _ = pk.token_logprobs(l1, d["y"], lse_low=low)
    d1 = pk.token_logprobs_grad(l1, d["y"], lse, ent, g, lse_low=low)
    d0 = pk.adjust_logits_grad(d1, l0, **kw)
    dh, dw2, _ = pk.linear_grad(d0, h, d["w2"])
    dy, dw1, dc1 = pk.linear_grad(dh, y, d["w1"], z, "gelu")
    dx, dw, db = pk.layer_norm_grad(dy, d["x"], d["w"], m, r)
    return lp, dict(x=dx + dh, w=dw, b=db, w1=dw1, c1=dc1, w2=dw2)


def _autograd(d, leaves):
    t = torch()
    y, _, _ = pk.layer_norm(leaves["x"], leaves["w"], leaves["b"])
    h = pk.linear(y, leaves["w1"], leaves["c1"], "gelu", leaves["x"], dtype=t.bfloat16)
    l0 = pk.linear(h, leaves["w2"])
    l1 = pk.adjust_logits(l0, tokens=d["tokens"], offsets=d["offsets"], repetition=d["rep"], allowed=d["allowed"],
                          mask=d["mask"])
    return pk.token_logprobs(l1, d["y"])[0]


@pytest.mark.parametrize("T,D,V", [(3, 40, 70), (65, 96, 333), (300, 264, 1001)])
def test_chain(T, D, V):
    t = torch()
    note(f"chain {T}x{D}x{V}")
    d = _data(T, D, V, T + V)
    # (rows whose token is forbidden have log probability -inf: none here)
    d["allowed"][:, :] = -1
    d["allowed"][0, 0] = -2
    d["y"].clamp_(min=1)
    g = t.randn(T, device="cuda")
    lp, want = _by_hand(d, g)
    assert t.isfinite(lp).all()
    leaves = {k: d[k].clone().requires_grad_() for k in want}
    out = _autograd(d, leaves)
    assert t.equal(out, lp)
    out.backward(g)
    for k in want:
        if k == "x":                       # (the residual's and the norm's, added by autograd in either order)
            assert t.equal(leaves[k].grad, want[k])
        else:
            assert t.equal(leaves[k].grad, want[k]), k


def _captured(call):
    t = torch()
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        call()
    t.cuda.current_stream().wait_stream(side)
    t.cuda.synchronize()
    g = t.cuda.CUDAGraph()
    with t.cuda.graph(g):
        out = call()
    return g, out


@pytest.mark.parametrize("T,D,V", [(1, 512, 1000), (70, 264, 333), (260, 1001, 777)])
def test_graph_replays(T, D, V):
    t = torch()
    note(f"chain captured {T}x{D}x{V}")
    d = _data(T, D, V, T)
    d["allowed"].fill_(-1)
    g = t.randn(T, device="cuda")

    def call():
        lp, grads = _by_hand(d, g)
        return (lp,) + tuple(grads.values())

    graph, out = _captured(call)
    for seed in (T, 5, 6):
        fresh = _data(T, D, V, seed)
        n = min(len(fresh["tokens"]), len(d["tokens"]))
        for k in d:
            if k == "tokens":
                d[k][:n] = fresh[k][:n]
            elif k not in ("offsets", "allowed"):
                d[k].copy_(fresh[k])
        want = [o.clone() for o in call()]
        for o in out:
            o.fill_(3)
        t.cuda.synchronize()
        graph.replay()
        t.cuda.synchronize()
        for a, b in zip(out, want):
            assert t.equal(a, b)


def test_graph_of_autograd():
    t = torch()
    note("autograd's chain captured")
    T, D, V = 70, 136, 333
    d = _data(T, D, V, 9)
    d["allowed"].fill_(-1)
    g = t.randn(T, device="cuda")
    leaves = {k: d[k].clone().requires_grad_() for k in ("x", "w", "b", "w1", "c1", "w2")}

    def call():
        out = _autograd(d, leaves)
        return (out.detach(),) + t.autograd.grad(out, list(leaves.values()), g)

    graph, out = _captured(call)
    for seed in (9, 10):
        fresh = _data(T, D, V, seed)
        with t.no_grad():
            for k, v in leaves.items():
                v.copy_(fresh[k])
                d[k].copy_(fresh[k])
        lp, want = _by_hand(d, g)
        graph.replay()
        t.cuda.synchronize()
        assert t.equal(out[0], lp)
        for a, k in zip(out[1:], leaves):
            assert t.equal(a, want[k]), k


def test_two_streams_at_once():
    t = torch()
    note("chains on two streams")
    a, b = _data(90, 264, 500, 1), _data(130, 136, 700, 2)
    ga, gb = t.randn(90, device="cuda"), t.randn(130, device="cuda")
    want = _by_hand(a, ga), _by_hand(b, gb)
    t.cuda.synchronize()
    s1, s2 = t.cuda.Stream(), t.cuda.Stream()
    for _ in range(5):
        with t.cuda.stream(s1):
            ra = _by_hand(a, ga)
        with t.cuda.stream(s2):
            rb = _by_hand(b, gb)
        t.cuda.synchronize()
        for got, ref in ((ra, want[0]), (rb, want[1])):
            assert t.equal(got[0].nan_to_num(), ref[0].nan_to_num())
            for k in got[1]:
                assert t.equal(got[1][k].nan_to_num(), ref[1][k].nan_to_num())


def test_given_workspaces_and_outputs():
    """A workspace larger than needed, filled with NaN, and outputs that are the
    caller's: the same results, and nothing beyond the outputs touched."""
    t = torch()
    note("given workspaces")
    M, K, N = 70, 1001, 264
    g = t.Generator().manual_seed(3)
    x, w = (t.randn((r, K), generator=g).bfloat16().cuda() for r in (M, N))
    dy = t.randn((M, N), generator=g).cuda()
    want, grads = pk.linear(x, w), pk.linear_grad(dy, x, w)
    ws = t.full((pk.linear_workspace(M, K, N).numel() + 512,), 255, dtype=t.uint8, device="cuda")
    assert t.equal(pk.linear(x, w, ws=ws), want)
    ws = t.full((pk.linear_grad_workspace(M, K, N).numel() + 512,), 255, dtype=t.uint8, device="cuda")
    tail = ws[-512:].clone()
    for a, b in zip(pk.linear_grad(dy, x, w, ws=ws), grads):
        assert t.equal(a, b)
    assert t.equal(ws[-512:], tail)
    _, m, r = pk.layer_norm(x, None)
    d = t.randn((M, K), generator=g).cuda()
    grads = pk.layer_norm_grad(d, x, None, m, r)
    ws = t.full((pk.layer_norm_grad_workspace(M, K).numel() + 512,), 255, dtype=t.uint8, device="cuda")
    for a, b in zip(pk.layer_norm_grad(d, x, None, m, r, ws=ws), grads):
        assert t.equal(a, b)
    assert t.equal(ws[-512:], tail)
    with pytest.raises(pk.ProfkError, match="needed"):
        pk.linear_grad(dy, x, w, ws=ws[:16])


def test_selection_after_masks():
    """The largest logits of an adjusted row are those of its allowed tokens."""
    t = torch()
    note("topk_rows of adjusted logits")
    T, V, k = 20, 5000, 7
    d = _data(T, 8, V, 4)
    x = t.randn((T, V), generator=t.Generator().manual_seed(1)).cuda()
    y = pk.adjust_logits(x, d["tokens"], d["offsets"], repetition=d["rep"], allowed=d["allowed"], mask=d["mask"])
    vals, idx, _ = pk.topk_rows(y, k)
    host, words = y.double().cpu().numpy(), d["allowed"].cpu().numpy().astype(np.int64) & 0xFFFFFFFF
    for r in range(T):
        order = np.lexsort((np.arange(V), -host[r]))[:k]
        got = idx.view(T, k)[r].cpu().numpy()
        assert (got == order).all()
        m = int(d["mask"][r])
        if m >= 0:
            assert ((words[m][got // 32] >> (got % 32)) & 1 == 1).all()
    _, _, _, top, at = pk.token_logprobs(y, d["y"], k)
    assert t.equal(at, idx.view(T, k).to(at.dtype))


def test_example():
    import train_head as ex
    t = torch()
    note("examples/train_head.py")
    r = ex.main(["--vocab", "333", "--dim", "72", "--rows", "200", "--steps", "3"])
    assert all(np.isfinite(v) for v in r["history"])
    assert r["free"].shape == (4, 7) and (r["even"][:, 1:] % 2 == 0).all()
    # its gradients, of the loss with penalties, are the calls' own
    p = ex.parameters(333, 72, 5, t.device("cuda"))
    tokens = t.arange(30, device="cuda") * 11 % 333
    history = (tokens.repeat(30), t.arange(31, device="cuda") * 30)
    rep = t.full((30,), 1.4, device="cuda")
    ex.loss(p, tokens, tokens + 1, history, repetition=rep).backward()
    x = p["embed"].detach()[tokens]
    q = {k: v.detach() for k, v in p.items()}
    y, m, s = pk.layer_norm(x, q["n1"], q["b1"])
    z = t.empty_like(x)
    h = pk.linear(y, q["w1"], q["c1"], "gelu", x, dtype=t.bfloat16, pre=z)
    y2, m2, s2 = pk.layer_norm(h, q["n2"], q["b2"])
    l0 = pk.linear(y2, q["w2"], q["c2"])
    l1 = pk.adjust_logits(l0, *history, repetition=rep)
    low = t.empty(30, device="cuda")
    _, ent, lse, _, _ = pk.token_logprobs(l1, tokens + 1, lse_low=low)
    g = t.full((30,), -1 / 30, device="cuda")
    d0 = pk.adjust_logits_grad(pk.token_logprobs_grad(l1, tokens + 1, lse, ent, g, lse_low=low), l0, *history, None, rep)
    dy2, dw2, dc2 = pk.linear_grad(d0, y2, q["w2"])
    dh, dn2, db2 = pk.layer_norm_grad(dy2, h, q["n2"], m2, s2)
    _, dw1, dc1 = pk.linear_grad(dh, y, q["w1"], z, "gelu")
    for k, want in dict(w2=dw2, c2=dc2, n2=dn2, b2=db2, w1=dw1, c1=dc1).items():
        got = p[k].grad
        # (the mean's 1 / 30 may be rounded another way: a unit in its last place)
        assert (got.double() - want.double()).norm() <= 2.0 ** -8 * want.double().norm(), k
