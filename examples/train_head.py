"""Train a small head and continue sequences with it under penalties.

The path of a language model's last block on synthetic tokens: an embedding, layer
norm, a dense layer with gelu and the residual stream in its epilogue, layer norm,
the unembedding, and the log probability of the next token, each with its
gradient through autograd; then, token by token, penalties for what was said, a
bias and a grammar's mask on the logits before the most probable token is taken.

    python examples/train_head.py [--vocab 1000] [--dim 128] [--rows 1024] [--steps 20]
"""

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2608_12573_amd as pk  # noqa: E402


def parameters(vocab, dim, seed, device):
    """bf16 weights and fp32 scales, shifts and biases, all trained."""
    g = torch.Generator(device=device).manual_seed(seed)

    def w(*shape):
        return (torch.randn(shape, generator=g, device=device) / dim ** 0.5).bfloat16().requires_grad_()

    def f(n, value):
        return torch.full((n,), value, device=device).requires_grad_()

    return dict(embed=w(vocab, dim), n1=f(dim, 1.0), b1=f(dim, 0.0), w1=w(dim, dim), c1=f(dim, 0.0), n2=f(dim, 1.0),
                b2=f(dim, 0.0), w2=w(vocab, dim), c2=f(vocab, 0.0))


def logits(p, tokens):
    """fp32 [T, V] for the token that follows each of [T]."""
    x = p["embed"][tokens]
    y, _, _ = pk.layer_norm(x, p["n1"], p["b1"])
    x = pk.linear(y, p["w1"], p["c1"], activation="gelu", residual=x, dtype=torch.bfloat16)
    y, _, _ = pk.layer_norm(x, p["n2"], p["b2"])
    return pk.linear(y, p["w2"], p["c2"])


def loss(p, tokens, following, history=None, **penalties):
    """Minus the mean log probability of `following`, under the penalties with
    which it was sampled."""
    x = logits(p, tokens)
    if history is not None:
        x = pk.adjust_logits(x, *history, **penalties)
    return -pk.token_logprobs(x, following)[0].mean()


def continue_tokens(p, start, steps, repetition, frequency, bias=None, allowed=None):
    """Each of [R] tokens continued by `steps` most probable ones; allowed: masks
    of tokens, or None."""
    R = len(start)
    said = start[:, None]
    with torch.no_grad():
        for _ in range(steps):
            x = logits(p, said[:, -1])
            offsets = torch.arange(R + 1, device=start.device) * said.shape[1]
            x = pk.adjust_logits(x, said.reshape(-1), offsets, repetition=repetition, frequency=frequency, bias=bias,
                                 allowed=allowed, out=x)
            _, best, _ = pk.topk_rows(x, 1)
            said = torch.cat([said, best.view(R, 1)], dim=1)
    return said


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--rows", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--lr", type=float, default=0.5)
    a = ap.parse_args(argv)
    dev = torch.device("cuda", torch.cuda.current_device())
    p = parameters(a.vocab, a.dim, 1, dev)
    g = torch.Generator(device=dev).manual_seed(2)
    tokens = torch.randint(a.vocab, (a.rows,), generator=g, device=dev)
    following = (tokens * 7 + 3) % a.vocab
    history = []
    for _ in range(a.steps):
        value = loss(p, tokens, following)
        history.append(value.item())
        value.backward()
        with torch.no_grad():
            for t in p.values():
                t -= a.lr * t.grad
                t.grad = None
    print(f"loss {history[0]:.4f} -> {history[-1]:.4f} in {a.steps} steps")
    start = tokens[:4]
    words = -(-a.vocab // 32)
    even = torch.full((1, words), 0x55555555, dtype=torch.int32, device=dev)
    one = torch.ones(4, device=dev)
    free = continue_tokens(p, start, 6, 1.3 * one, 0.5 * one)
    said = continue_tokens(p, start, 6, 1.3 * one, 0.5 * one, allowed=even)
    print("continued:", free.tolist())
    print("with even tokens alone:", said.tolist())
    return dict(history=history, free=free, even=said)


if __name__ == "__main__":
    main()
