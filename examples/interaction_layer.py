"""One interaction layer of an equivariant network: the tensor product on the edges, then the feed-forward block
on the invariant channels of the nodes, as a training step with 8-bit checkpoints and as inference in 8 bits.

    python examples/interaction_layer.py

Training: the messages are SpinGTP products; their invariant part (spin 0, degree 0) is summed onto the nodes,
added to the nodes' state and normalised (``rms_norm``), and passes the gated block (``gated``) and a
projection.  What the backward pass needs of the coefficients and of the block is kept in 8 bits
(``pack8``, ``save="8bit"``), a quarter of the fp32 coefficients' memory.
Inference: the same block from weights packed once; each operator hands the next one 8-bit blocks.
"""

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_01408_amd as sg  # noqa: E402
from paper_2607_01408_amd import workloads  # noqa: E402

INVARIANT = (workloads.SPINS.index(0), 0)  # of a unit's coefficients: spin 0, degree 0


def weights(C, F, seed=1, device="cuda"):
    """Gain and the three matrices of the block, bf16."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)

    def draw(n, k):
        return (torch.randn((n, k), generator=g, device=device) / k**0.5).bfloat16()

    return dict(gain=torch.ones(C, device=device), gate=draw(F, C), up=draw(F, C), down=draw(C, F))


def sum_onto_nodes(messages, receivers, nodes):
    """[nodes, C] sums of the invariant part of the edges' messages."""
    part = messages[:, :, INVARIANT[0], INVARIANT[1]].float()
    return torch.zeros((nodes, part.shape[1]), device=part.device).index_add_(0, receivers, part)


def train_step(plan, x1, x2, receivers, state, w, grad_out):
    """(new state, gradients) of one layer for a loss with dLoss/d(new state) = grad_out.

    x1, x2 [N, C, 3, (L+1)^2] fp32; state, grad_out [nodes, C] bf16."""
    N, C = x1.shape[:2]
    # forward
    kept = [sg.pack8(x.view(N, -1)) for x in (x1, x2)]
    node = sum_onto_nodes(plan.forward(x1, x2), receivers, len(state)).bfloat16()
    y, h, rstd = sg.rms_norm(node, w["gain"], residual=state)
    hidden, saved = sg.gated(y, w["gate"], w["up"], save="8bit")
    new = h + hidden @ w["down"].t()
    # backward
    grad_hidden = grad_out @ w["down"]
    grads = {"down": grad_out.t() @ hidden}
    grad_y, grads["gate"], grads["up"] = sg.gated_backward(grad_hidden, saved, w["gate"], w["up"])
    grads["state"], grads["gain"] = sg.rms_norm_backward(grad_y, h, rstd, w["gain"], grad_h=grad_out)
    grad_messages = torch.zeros((N, C) + plan.shape_out, device=x1.device)
    grad_messages[:, :, INVARIANT[0], INVARIANT[1]] = grads["state"].float()[receivers]
    again = [sg.unpack8(b, dtype=torch.float32).view(x.shape) for b, x in zip(kept, (x1, x2))]
    grads["x1"], grads["x2"] = plan.backward(*again, grad_messages)
    return new, grads


def pack_weights(w):
    """The block's weights for inference, packed once."""
    return dict(gain=w["gain"], **{k: sg.pack8(w[k]) for k in ("gate", "up", "down")})


def infer(node, state, w8):
    """New state from the nodes' invariant messages, everything between the operators in 8 bits."""
    y, h, _ = sg.rms_norm(node, w8["gain"], residual=state, out8=True)
    hidden, _ = sg.gated(y, w8["gate"], w8["up"], out8=True)
    return h + sg.matmul8(hidden, w8["down"])


def main():
    nodes, N, C, F, L = 320, 4000, 64, 256, 2
    x1, x2, _ = workloads.make_pair("small", N=N, C=C)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    receivers = torch.randint(nodes, (N,), generator=g, device="cuda")
    state, grad_out = (torch.randn((nodes, C), generator=g, device="cuda").bfloat16() for _ in range(2))
    w = weights(C, F)
    plan = sg.Plan(L, L, L, workloads.SPINS, "fp32")
    new, grads = train_step(plan, x1, x2, receivers, state, w, grad_out)
    node = sum_onto_nodes(plan.forward(x1, x2), receivers, nodes).bfloat16()
    served = infer(node, state, pack_weights(w))
    off = float((served.float() - new.float()).norm() / new.float().norm())
    print(f"{N} edges, {nodes} nodes, {C} channels: gradients " +
          ", ".join(f"{k} {float(v.float().norm()):.3g}" for k, v in grads.items()))
    print(f"inference in 8 bits against the training forward: relative difference {off:.3g}")


if __name__ == "__main__":
    main()
