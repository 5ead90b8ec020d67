"""A drafter distilled from a target's own rollout, on the library's operators alone.

The target is a random bigram model: the logits after a token are its embedding times a head.  Each step

  1. embeds the running sequences' last tokens (alr_embed), takes the target's logits with the head
     (alr_gemm), keeps the label, its top 8 logits and the mass of the rest (alr_top_logits), and draws
     the next tokens (alr_sample_tokens);
  2. embeds the same tokens with the drafter's table, takes its logits with the same head, and has
     the loss and the logit gradient in one pass (alr_distill_fwd_bwd, the gradient over the logits);
  3. carries the gradient back: dH = G W^T (alr_gemm), the table's gradient by token
     (alr_embed_grad), and a step of gradient descent.

The drafter's loss falls towards the label's entropy, the least it can be.

  python examples/distil_drafter.py [--steps 200] [--rows 512] [--vocab 4096] [--dim 256]
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_38795_gb300 import alr  # noqa: E402


def train(steps=200, rows=512, vocab=4096, dim=256, lr=150.0, seed=0, report=print):
    """Returns the mean KL divergence of the first and of the last ten steps."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    bf = torch.bfloat16
    head = r(vocab, dim).to(bf) * dim ** -0.5                 # W^T, K-major for alr_gemm
    head_t = head.t().contiguous()                            # W, for dH = G W^T
    target, drafter = (r(vocab, dim) * 2.5).to(bf), torch.zeros(vocab, dim, device="cuda")
    K, N = 8, rows
    f = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    i = lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    token = torch.randint(0, vocab, (N,), generator=g, device="cuda", dtype=torch.int32)
    hidden, z_t, z_d, dH = torch.empty(N, dim, dtype=bf, device="cuda"), f(N, vocab), f(N, vocab), f(N, dim)
    label = dict(top_val=f(N, K), top_idx=i(N, K), lse_rest=f(N))
    drawn = dict(token=i(N), prob=f(N))
    out = dict(loss_row=f(N), ent_row=f(N), lse=f(N), lse_rest=f(N), loss_total=f(1), weight_sum=f(1))
    grad, G = f(vocab, dim), torch.empty(N, vocab, dtype=bf, device="cuda")
    ws = torch.empty(alr.alr_embed_grad_workspace_size(vocab, dim, N), dtype=torch.uint8, device="cuda")
    temperature, top_p = torch.full((N,), 1.0, device="cuda"), torch.full((N,), 0.95, device="cuda")
    kl = []
    for step in range(steps):
        u = torch.randint(-(1 << 31), 1 << 31, (N,), generator=g, device="cuda",
                          dtype=torch.int64).to(torch.int32)
        # the target's step of the rollout: label and next token
        alr.alr_embed(target, token, hidden)
        alr.alr_gemm(hidden, head, z_t, N, vocab, dim)
        alr.alr_top_logits(z_t, K, label)
        alr.alr_sample_tokens(z_t, u, drawn, temperature=temperature, top_p=top_p)
        # the drafter's: loss, gradient of its logits, of its hidden states, of its table
        alr.alr_embed(drafter.to(bf), token, hidden)
        alr.alr_gemm(hidden, head, z_d, N, vocab, dim)
        alr.alr_distill_fwd_bwd(z_d, label["top_val"], label["top_idx"], out, z_d, rest=label["lse_rest"])
        G.copy_(z_d)
        alr.alr_gemm(G, head_t, dH, N, dim, vocab)
        alr.alr_embed_grad(dH, token, grad, ws)
        drafter.add_(grad, alpha=-lr)
        token.copy_(drawn["token"])
        kl.append(out["loss_row"].mean() - out["ent_row"].mean())
        if report and (step % 50 == 0 or step == steps - 1):
            report(f"step {step:4d}: loss {out['loss_total'].item():.4f}, above the label's entropy "
                   f"{kl[-1].item():.4f}")
    assert alr.alr_device_status() == alr.ALR_OK
    kl = torch.stack(kl).cpu()
    return kl[:10].mean().item(), kl[-10:].mean().item()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--rows", type=int, default=512)
    ap.add_argument("--vocab", type=int, default=4096)
    ap.add_argument("--dim", type=int, default=256)
    a = ap.parse_args()
    train(a.steps, a.rows, a.vocab, a.dim)
