"""A layer's whole training step in one HIP graph: connect with a norm in front of its branch, the gradients, and the
update of the coefficients' matrix, replayed between eager work, against the same eagerly, bit for bit."""
import pytest
import torch

import paper_2606_07574_amd as b4

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("steps", [5, 8])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,C", [(4, 72), (8, 64)])
def test_training_step(n, C, dtype, steps):
    B, R = 50, n * n + 2 * n
    g = torch.Generator(device="cuda").manual_seed(n)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)
    data = [(normal(B, n, C).to(dtype), normal(B, n, C).to(dtype)) for _ in range(4)]
    W0, M0 = (normal(R, n * C) / (n * C) ** 0.5).to(dtype), torch.zeros(R, n * C, device="cuda")
    small = [torch.ones(3, device="cuda"), 0.1 * normal(R), (1 + 0.1 * normal(C)), 0.1 * normal(C)]

    def step(X, dY, W, M, small, lr):
        leaves = [t.detach().requires_grad_() for t in (X, W, *small)]
        Y = b4.connect(*leaves[:4], torch.tanh, norm=leaves[4:])
        grads = torch.autograd.grad(Y, leaves, dY)
        b4.orth_step(W, grads[1], M, lr, decay=0.1, steps=steps)
        return (Y.detach(), *grads)

    def state():
        return W0.clone(), M0.clone(), [t.clone() for t in small], torch.tensor(0.1, device="cuda")

    X, dY = (t.clone() for t in data[0])
    held, spare, eager = state(), state(), state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(X, dY, *spare)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(X, dY, *held)
    for turn, (x, dy) in enumerate(data):
        X.copy_(x)
        dY.copy_(dy)
        for s in (held, eager):
            s[3].fill_(0.1 / (turn + 1))
        want = step(x, dy, *eager)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((*outs, held[0], held[1]), (*want, eager[0], eager[1])):
            assert torch.equal(a, b), turn
        for o in outs:
            o.fill_(float("nan"))
