"""Train an unembedding, hold it in 4 bits, and score tokens with it.

The path from a language model's last hidden state to its answer, on synthetic
hidden states: logits x W^T of a vocabulary, the log probability of each row's
token with the entropy and the most probable alternatives, their gradient for
training, and W as 4-bit microscaled values for serving.

    python examples/score_tokens.py [--vocab 4096] [--dim 256] [--rows 2048] [--steps 20]
"""

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2608_12573_amd as pk  # noqa: E402


def data(rows, vocab, dim, seed, device):
    """Hidden states and the tokens that a fixed unembedding samples for them;
    one row in ten is padding and has no token."""
    g = torch.Generator(device=device).manual_seed(seed)
    teacher = torch.randn((vocab, dim), generator=torch.Generator(device=device).manual_seed(1), device=device)
    x = torch.randn((rows, dim), generator=g, device=device)
    p = torch.softmax(x @ teacher.t() * (3.0 / dim ** 0.5), dim=1)
    y = torch.multinomial(p, 1, generator=g)[:, 0]
    y[torch.rand(rows, generator=g, device=device) < 0.1] = -1
    return x.bfloat16(), y


def train(w, x, y, steps, lr, entropy_weight):
    """Gradient descent on -mean log probability - entropy_weight mean entropy
    over the rows with a token, of the fp32 master weights w in place; returns
    each step's mean log probability."""
    given = (y >= 0).float()
    g_lp = given / -given.sum()
    g_h = given * (-entropy_weight / given.sum())
    out = pk.token_logprobs_outputs(x.shape[0], 0, x.device)
    ws = pk.token_logprobs_workspace(x.shape[0], w.shape[0], 0, x.device)
    low = torch.empty(x.shape[0], device=x.device)
    d = torch.empty((x.shape[0], w.shape[0]), device=x.device)
    xf, m, history = x.float(), torch.zeros_like(w), []
    for _ in range(steps):
        logits = xf @ w.t()
        lp, h, lse, _, _ = pk.token_logprobs(logits, y, ws=ws, out=out, lse_low=low)
        history.append((lp.sum() / given.sum()).item())
        pk.token_logprobs_grad(logits, y, lse, h, g_lp, g_h, out=d, lse_low=low)
        m.mul_(0.9).add_(d.t() @ xf)
        w.sub_(m, alpha=lr)
    return history


def score(logits, y, n_top):
    """Mean log probability of the tokens, and the rows' alternatives."""
    lp, h, _, top, idx = pk.token_logprobs(logits, y, n_top)
    return lp.sum().item() / int((y >= 0).sum()), h.mean().item(), top, idx


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--vocab", type=int, default=4096)
    ap.add_argument("--dim", type=int, default=256)
    ap.add_argument("--rows", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--lr", type=float, default=0.3)
    ap.add_argument("--top", type=int, default=5)
    a = ap.parse_args(argv)
    dev = torch.device("cuda", torch.cuda.current_device())
    x, y = data(a.rows, a.vocab, a.dim, 2, dev)
    w = torch.zeros((a.vocab, a.dim), device=dev)
    history = train(w, x, y, a.steps, a.lr, entropy_weight=0.01)
    print(f"training: mean log probability {history[0]:.4f} -> {history[-1]:.4f} in {a.steps} steps")

    codes, scales = pk.mx4_quantize(w)               # once, for serving
    full = score(x.float() @ w.t(), y, a.top)
    four = score(pk.mx4_linear(x, codes, scales), y, a.top)
    one = score(pk.mx4_linear(x[:1], codes, scales), y[:1].clamp(min=0), a.top)
    agree = (full[3][:, 0] == four[3][:, 0]).float().mean().item()
    print(f"weights: {w.numel() * 4} bytes in fp32, {codes.numel() + scales.numel()} in 4 bits")
    print(f"log probability {full[0]:.4f} in fp32, {four[0]:.4f} in 4 bits; entropy {full[1]:.4f}, {four[1]:.4f}; "
          f"the same first alternative in {100 * agree:.1f} % of rows")
    print("one row's alternatives:", [(int(i), round(float(v), 3)) for v, i in zip(one[2][0], one[3][0])])
    return dict(history=history, full=full, four=four, one=one, agree=agree)


if __name__ == "__main__":
    main()
