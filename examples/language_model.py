"""Replicas of a small language model trained with delayed averaging: the operators of the library in one loop.

K replicas predict the next token of synthetic sequences.  The weights of a replica are one row of the engine's arrays:

    | embedding table  V x D | hidden layer  H x D | output layer  V x H |

Every step looks the tokens' rows up in the weights (``Embedding.lookup``), runs the two layers (torch), writes the
table's gradient beside the layers' (``Embedding.gradient``), turns the layers' gradients into orthogonalised directions in place
(``Ortho.step``; the table keeps its gradient), and hands the array to the engine (``DaSGD.step``), which subtracts it
from every replica, snapshots, and blends the stale mean in.  Everything is enqueued on the engine's main stream.

    python examples/language_model.py [--steps 60] [--dtype bf16|f32]
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2006_00441_b200 import binding as B  # noqa: E402


def train(steps=60, K=4, V=512, D=128, H=256, T=1024, dtype=B.DASGD_BF16_MASTER_F32, lr=0.02, table_lr=4.0, tau=2, d=1, seed=0):
    """The mean loss of the replicas, step by step."""
    gen = torch.Generator("cuda").manual_seed(seed)
    n_table, n_hidden, n_out = V * D, H * D, V * H
    P = n_table + n_hidden + n_out
    eng = B.DaSGD(K, P, tau, d, xi=0.25, dtype=dtype, flags=B.DASGD_FLAG_ROTATE_SNAPSHOT | B.DASGD_FLAG_FUSE_MERGE)
    emb = B.Embedding(K, P, 0, V, D, scale=D ** 0.5, max_tokens=T)
    ortho = B.Ortho(K, P, [(n_table, H, D, (H / D) ** 0.5), (n_table + n_hidden, V, H, (V / H) ** 0.5)], dtype=dtype, momentum=0.9)
    w0 = torch.cat([0.5 * D ** -0.5 * torch.randn(n_table, generator=gen, device="cuda"),
                    D ** -0.5 * torch.randn(n_hidden, generator=gen, device="cuda"),
                    0.1 * H ** -0.5 * torch.randn(n_out, generator=gen, device="cuda")])
    eng.set_state(w0)
    follows = torch.randperm(V, generator=gen, device="cuda")   # the rule to learn: which token follows which
    g = torch.zeros(K, P, dtype=eng.gdtype, device="cuda")
    m = torch.zeros(K, P, device="cuda")
    losses = []
    torch.cuda.synchronize()
    with torch.cuda.stream(eng.main):
        for _ in range(steps):
            tokens = torch.randint(0, V, (K, T), generator=gen, device="cuda")
            tokens[:, -T // 16:] = -1                            # padding: zero rows, no gradient
            w = eng.w if eng.w_lp is None else eng.w_lp
            hidden = w[:, n_table:n_table + n_hidden].view(K, H, D).detach().requires_grad_()
            out = w[:, n_table + n_hidden:].view(K, V, H).detach().requires_grad_()
            x = emb.lookup(w, tokens).requires_grad_()
            logits = torch.relu(x @ hidden.mT) @ out.mT
            target = torch.where(tokens >= 0, follows[tokens.clamp(min=0)], -100)
            loss = F.cross_entropy(logits.float().view(-1, V), target.view(-1), ignore_index=-100, reduction="sum") / (target >= 0).sum() * K
            dx, dh, do = torch.autograd.grad(loss, (x, hidden, out))
            g[:, n_table:n_table + n_hidden] = dh.reshape(K, -1)
            g[:, n_table + n_hidden:] = do.reshape(K, -1)
            emb.gradient(dx * (table_lr / lr), tokens, g)        # the engine has one rate: the table's own is in its gradient
            ortho.step(g, m)
            eng.step(g, lr)
            losses.append(loss.detach() / K)
    eng.sync()
    ortho.sync()
    losses = torch.stack(losses).tolist()
    eng.close()
    ortho.close()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = ap.parse_args()
    for i, loss in enumerate(train(a.steps, dtype=B.DASGD_F32 if a.dtype == "f32" else B.DASGD_BF16_MASTER_F32)):
        if i % 5 == 0 or i + 1 == a.steps:
            print(f"step {i:4d}  loss {loss:.4f}")
