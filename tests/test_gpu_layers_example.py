"""The layer operators together: the example's network against the same network in 64 bits with torch's own gradients, its training with
and without checkpoints, and a step captured in a graph."""
import os
import sys

import pytest
import torch

from paper_2502_17846_amd import binding as B
from tests import ref_layers as ref

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import train_on_partitions as example  # noqa: E402

pytestmark = pytest.mark.gpu


def _plain_gradients(net, x, target):
    """Loss and gradients in 64 bits on the CPU, by torch's automatic differentiation."""
    params = {k: v.cpu().double().requires_grad_() for k, v in net.params.items()}
    rows, cols = ref.kept_entries(net.rowptr.cpu().numpy(), net.colidx.cpu().numpy(), net.labels.cpu().numpy())
    counts = torch.bincount(rows, minlength=net.n).clamp(min=1).double().unsqueeze(1)

    def layer(h, name, residual, last=False):
        around = torch.zeros_like(h).index_add(0, rows, h[cols]) / counts
        z = torch.cat([h, around], 1) @ params[name + ".w"].T + params[name + ".bias"]
        if last:
            return z
        out = z * torch.sigmoid(z) + (h if residual else 0)
        out = out - out.mean(1, keepdim=True)
        return out * ((out * out).mean(1, keepdim=True) + 1e-5) ** -0.5 * params[name + ".gamma"] + params[name + ".beta"]

    h = layer(x.cpu().double(), "in", False)
    h = layer(h, "hidden", True)
    loss = -torch.log_softmax(layer(h, "out", False, True), 1).gather(1, target.cpu().unsqueeze(1)).mean()
    loss.backward()
    return loss.item(), {k: v.grad for k, v in params.items()}


def test_gradients_of_the_network():
    graph, x, target = example.problem(n=2_000, features=50, dtype=torch.float32)
    net = example.Network(graph, 50, 64, 4, torch.float32, checkpoints=False)
    loss, grads, _ = net.gradients(x, target)
    want_loss, want = _plain_gradients(net, x, target)
    # sums of at most 2,000 terms: 2^-24 * 2,000 = 1.2e-4 of the terms' sizes at the very worst, passed on through three layers; terms of
    # random signs come to a hundredth of that
    assert abs(loss.item() - want_loss) < 1e-5
    for name, g in want.items():
        assert (grads[name].cpu().double() - g).norm() < 1e-4 * g.norm(), name


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_training_with_checkpoints(kind):
    t = example.TYPES[kind]
    graph, x, target = example.problem(dtype=t)
    plain = example.Network(graph, x.shape[1], 128, 4, t, checkpoints=False)
    packed = example.Network(graph, x.shape[1], 128, 4, t, checkpoints=True)
    loss, want, _ = plain.gradients(x, target)
    same, grads, _ = packed.gradients(x, target)
    assert same.item() == loss.item()                     # the forward pass does not read them
    for name, g in want.items():
        # a value is off by at most 1/127 of its group's largest; these are sums over 10,000 rows of errors of either sign
        assert (grads[name] - g).norm() < 2.0 ** -5 * g.norm(), name
    losses = example.train(packed, x, target, 25)
    assert losses[0] > 1.0 and losses[-1] < 0.5 * losses[0], losses


def test_a_captured_step():
    graph, x, target = example.problem(n=3_000, features=64)
    net = example.Network(graph, 64, 64, 4, torch.bfloat16)
    w = net.params["in.w"].to(torch.bfloat16)
    gamma, dy = torch.ones(64, dtype=torch.bfloat16, device="cuda"), torch.ones((net.n, 64), dtype=torch.bfloat16, device="cuda")

    def step(v):
        around, counts = B.grem_neighbour_mean(net.rowptr, net.colidx, net.n, v, net.labels)
        out, z = B.grem_linear(v, w, b=around, act=B.ACT_GELU, residual=v, want_pre=True)
        kept = B.grem_checkpoint_pack(out)
        y, mean, rstd = B.grem_layer_norm(out, gamma)
        d, dgamma, dbeta = B.grem_layer_norm_backward(dy * y, kept, mean, rstd, gamma)
        da, db, dw, dbias = B.grem_linear_backward(d, B.grem_checkpoint_pack(v), w, b=B.grem_checkpoint_pack(around), act=B.ACT_GELU, pre=z)
        dx = B.grem_neighbour_mean_backward(net.rowptr, net.colidx, net.n, db, counts, net.labels)
        return y, da, dx, dw, dbias, dgamma, dbeta, B.grem_checkpoint_unpack(kept)

    fed = x.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(fed)
    torch.cuda.current_stream().wait_stream(side)
    graph_ = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph_):
        held = step(fed)
    for turn in range(4):
        fed.copy_(x * (turn + 1))
        want = [v.clone() for v in step(x * (turn + 1))]        # the program's own work between the replays
        graph_.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
