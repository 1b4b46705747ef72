"""The example layer (tensor product, norm, gated block, 8-bit checkpoints) against float64 autograd (GPU)."""

import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2607_01408_amd as sg  # noqa: E402
from paper_2607_01408_amd import dense_tensor_host, workloads  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("interaction_layer", os.path.join(ROOT, "examples", "interaction_layer.py"))
layer = importlib.util.module_from_spec(spec)
spec.loader.exec_module(layer)


def relative(got, ref):
    return float((got.double() - ref).norm() / ref.norm())


@pytest.mark.parametrize("nodes,N,C,F", [(30, 200, 16, 48), (7, 33, 24, 200)])
def test_layer(nodes, N, C, F):
    L = 2
    x1, x2, _ = workloads.make_pair("small", N=N, C=C)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    receivers = torch.randint(nodes, (N,), generator=g, device="cuda")
    state, grad_out = (torch.randn((nodes, C), generator=g, device="cuda").bfloat16() for _ in range(2))
    w = layer.weights(C, F)
    plan = sg.Plan(L, L, L, workloads.SPINS, "fp32")
    new, grads = layer.train_step(plan, x1, x2, receivers, state, w, grad_out)

    T = torch.as_tensor(dense_tensor_host(L, L, L), device="cuda")
    p = {k: v.double().requires_grad_() for k, v in dict(w, x1=x1, x2=x2, state=state).items()}
    flat = [p[k].reshape(N * C, -1) for k in ("x1", "x2")]
    product = torch.zeros((N * C, T.shape[2]), dtype=torch.float64, device="cuda")
    for k in range(T.shape[0]):  # sum over the first input's coefficients
        product = product + flat[0][:, k : k + 1] * (flat[1] @ T[k])
    messages = product.view(N, C, 3, -1)[:, :, layer.INVARIANT[0], layer.INVARIANT[1]]
    node = torch.zeros((nodes, C), dtype=torch.float64, device="cuda").index_add(0, receivers, messages)
    h = node + p["state"]
    y = h * (h.pow(2).mean(-1, keepdim=True) + 1e-6).rsqrt() * p["gain"]
    gate, up = y @ p["gate"].t(), y @ p["up"].t()
    out = h + (gate * torch.sigmoid(gate) * up) @ p["down"].t()
    out.backward(grad_out.double())

    # bf16 on the way forward: a handful of roundings of 2^-9 each
    assert relative(new, out.detach()) <= 8 * 2.0**-9
    # gradients that pass an 8-bit checkpoint: rounding to e4m3 is 2^-4 of an element at most and 2^-4 / sqrt(3) in
    # the root mean square; at most two checkpointed factors meet in a term
    for k in ("gate", "up", "gain", "state", "x1", "x2"):
        assert relative(grads[k], p[k].grad) <= 2 * 2.0**-4, k
    assert relative(grads["down"], p["down"].grad) <= 8 * 2.0**-9

    # inference: three 8-bit operands of a product each, two products in turn, added to the state
    served = layer.infer(node.detach().bfloat16(), state, layer.pack_weights(w))
    assert relative(served, out.detach()) <= 4 * 2.0**-4
    torch.cuda.synchronize()


def test_example_runs(capsys):
    layer.main()
    assert "relative difference" in capsys.readouterr().out
