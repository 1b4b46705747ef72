"""One interaction layer of an equivariant network: the tensor product on the edges, then the feed-forward block
on the invariant channels of the nodes, as a training step with 8-bit checkpoints and update and as inference in 8 bits.

    python examples/interaction_layer.py

Training: the messages are SpinGTP products; their invariant part (spin 0, degree 0) is summed onto the nodes
(``embedding_backward``, the gradient of the lookup that hands the nodes' gradients back to the edges), added to
the nodes' state and normalised (``rms_norm``), and passes the gated block (``gated``) and a projection onto the
residual stream (``linear``).  What the backward pass needs of the coefficients and of the block is kept in 8 bits
(``pack8``, ``save="8bit"``), a quarter of the fp32 coefficients' memory.  ``adamw`` updates fp32 weights, with 8-bit
states, and the bf16 copies that the layer reads.
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
    """[nodes, C] sums of the invariant part of the edges' messages; receivers: the edges' nodes, or their SortedIndex."""
    part = messages[:, :, INVARIANT[0], INVARIANT[1]].contiguous()
    return sg.embedding_backward(part, receivers, nodes)


def train_step(plan, x1, x2, receivers, state, w, grad_out):
    """(new state, gradients) of one layer for a loss with dLoss/d(new state) = grad_out.

    x1, x2 [N, C, 3, (L+1)^2] fp32; state, grad_out [nodes, C] bf16."""
    N, C = x1.shape[:2]
    # forward
    kept = [sg.pack8(x.view(N, -1)) for x in (x1, x2)]
    edges = sg.sort_index(receivers, len(state))  # once for as many layers as have these edges
    node = sum_onto_nodes(plan.forward(x1, x2), edges, len(state)).bfloat16()
    y, h, rstd = sg.rms_norm(node, w["gain"], residual=state)
    hidden, saved = sg.gated(y, w["gate"], w["up"], save="8bit")
    new, last = sg.linear(hidden, w["down"], residual=h, save="same")
    # backward
    grad_hidden, grad_down, _ = sg.linear_backward(grad_out, last, w["down"], need_bias=False)
    grads = {"down": grad_down}
    grad_y, grads["gate"], grads["up"] = sg.gated_backward(grad_hidden, saved, w["gate"], w["up"])
    grads["state"], grads["gain"] = sg.rms_norm_backward(grad_y, h, rstd, w["gain"], grad_h=grad_out)
    grad_messages = torch.zeros((N, C) + plan.shape_out, device=x1.device)
    grad_messages[:, :, INVARIANT[0], INVARIANT[1]] = sg.embedding(grads["state"], receivers).float()
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
    return sg.linear(hidden, w8["down"], residual=h)[0]


class Update:
    """fp32 weights and their AdamW states in 8 bits; ``step`` updates them and the layer's weights."""

    def __init__(self, w):
        self.w = w
        self.master = {k: v.float().clone() for k, v in w.items()}
        self.states = {k: sg.adamw_state(v, bits=8) for k, v in self.master.items()}
        self.steps = 0

    def step(self, grads, lr=1e-3):
        self.steps += 1
        names = list(self.master)
        m, v = zip(*(self.states[k] for k in names))
        sg.adamw([self.master[k] for k in names], [grads[k] for k in names], m, v, step=self.steps, lr=lr,
                 copies=[self.w[k] if self.w[k].dtype == torch.bfloat16 else None for k in names])
        for k in names:
            if self.w[k].dtype == torch.float32:
                self.w[k].copy_(self.master[k])


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
    update = Update(w)
    update.step(grads)
    after, _ = train_step(plan, x1, x2, receivers, state, w, grad_out)
    went = float(((after.float() - new.float()) * grad_out.float()).sum())
    print(f"one AdamW step moves the loss by {went:.3g}")


if __name__ == "__main__":
    main()
