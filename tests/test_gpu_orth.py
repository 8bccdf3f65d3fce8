"""GPU parity of the orthogonalisation (birkhoff4_orth) and of the update around it (birkhoff4_orth_step)
with float64, within what the stated roundings may do (tests/_orth.py)."""
import math

import pytest
import torch

import paper_2606_07574_amd as b4
from tests._orth import close, orth_ref

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def matrices(shape, dtype, seed, kind="mixed", size=1e-2):
    """Gradients: spread out, a few strong directions and a rest, or these alone (low rank)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)
    *lead, m, n = shape
    if kind == "spread":
        return (size * normal(*shape)).to(dtype)
    r = min(m, n, 8)
    strong = normal(*lead, m, r) * torch.exp(-0.3 * torch.arange(r, device="cuda")) @ normal(*lead, r, n)
    return (size * (strong + (0.3 * normal(*shape) if kind == "mixed" else 0))).to(dtype)


def check(G, label, **kw):
    print(label, flush=True)
    O = b4.orth(G, **kw)
    torch.cuda.synchronize()
    assert O.shape == G.shape and O.dtype == G.dtype
    ref, bound = orth_ref(G, split=G.dtype == F32, **kw)
    close(O, ref, bound, label)


# one value, one row, one column, fewer than a piece; the coefficients' matrices (24 and 80 rows); both
# sides of every tile and of the lines of 32 and 64; tall, wide and square; batches
SIZES = [(1, 1), (3, 1, 7), (9, 1), (2, 3, 5), (5, 8, 8), (24, 1000), (3, 80, 2056), (2, 500, 24), (79, 81), (81, 79), (80, 80),
         (4, 64, 64), (2, 65, 33), (128, 128), (129, 127), (127, 300), (2, 128, 256), (2, 200, 130), (257, 640), (513, 256),
         (384, 1001), (7, 96, 160), (1000, 300), (300, 1000), (2, 640, 640), (31, 100, 100), (200, 5000), (1100, 1100),
         # runs of 64 and 256 columns and what is left of them, every number of tiles of the narrow ones
         (16, 700), (3, 33, 1025), (48, 4100), (2, 50, 513), (300, 24, 1000), (40, 64, 8200), (70, 30001), (65000, 2, 3)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SIZES, ids=str)
def test_sizes(shape, dtype):
    check(matrices(shape, dtype, sum(shape)), f"{shape} {dtype}")


@pytest.mark.parametrize("kind", ["spread", "low"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(24, 777), (2, 200, 333), (512, 128)], ids=str)
def test_spectra(shape, dtype, kind):
    check(matrices(shape, dtype, 5, kind), f"{shape} {dtype} {kind}")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(24, 200), (3, 150, 140)], ids=str)
def test_steps_and_coefficients(shape, dtype):
    """One step to many, a triple for each step, and the cubic whose singular values go to one."""
    G = matrices(shape, dtype, 6, "spread")
    for steps in (1, 2, 3, 8):
        check(G, f"{steps} steps", steps=steps)
    schedule = [(4.0, -6.0, 2.5), (3.5, -5.0, 2.1), (1.875, -1.25, 0.375), (1.875, -1.25, 0.375)]
    check(G, "schedule", steps=4, coefs=schedule)
    check(G, "cubic", steps=25, coefs=(1.5, -0.5, 0.0))
    O = b4.orth(G, steps=25, coefs=(1.5, -0.5, 0.0)).double().reshape(-1, *shape[-2:])
    if shape[-2] > shape[-1]:
        O = O.transpose(1, 2)
    gram = O @ O.transpose(1, 2).contiguous()
    eye = torch.eye(gram.shape[1], dtype=torch.float64, device="cuda")
    # rows of length one whose values are rounded by half a step each
    assert (gram - eye).abs().max() < (1e-5 if dtype == F32 else 2 * 2.0 ** -8)


@pytest.mark.parametrize("shape", [(24, 200), (40, 40), (150, 260)], ids=str)
def test_sizes_of_values(shape):
    """Powers of two in front change nothing at all without eps; the far ends of fp32 are fine."""
    G = matrices(shape, F32, 7, "spread", 1.0)
    O = b4.orth(G, eps=0.0)
    for e in (-100, -20, 40, 120):
        assert torch.equal(b4.orth(G * 2.0 ** e, eps=0.0), O)
    check(G * 1e-7, "against eps", eps=1e-5)
    check(G * 2.0 ** -126, "below the smallest normal value", eps=0.0)
    assert (b4.orth(torch.zeros_like(G)) == 0).all()


@pytest.mark.parametrize("shape", [(24, 200), (3, 80, 5000), (200, 24), (150, 260)], ids=str)
def test_sizes_of_bf16_values(shape):
    """The same of bf16 values, whose squares leave fp32's range at both ends; and a matrix with a part that
    is far larger, or far smaller, than the rest."""
    G = matrices(shape, BF16, 7, "spread", 1.0)
    O = b4.orth(G, eps=0.0)
    assert O.isfinite().all()
    for e in (-100, -66, -20, 40, 66, 120):
        assert torch.equal(b4.orth(G * 2.0 ** e, eps=0.0), O), e
    check(G * 2.0 ** -126, "below the smallest normal value", eps=0.0)
    check(G * 2.0 ** -70, "against eps", eps=2.0 ** -66)
    for e in (-80, 100):
        part = G.clone()
        part[..., : shape[-1] // 2] *= 2.0 ** e
        check(part, f"a half 2^{e} times", eps=0.0)
    assert (b4.orth(torch.zeros_like(G)) == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 24, 333), (2, 150, 333), (100, 700)], ids=str)
def test_transpose(shape, dtype):
    """The transpose's result is the result's transpose, bit for bit but for narrow bf16 matrices, whose rows
    are taken as they lie (there half a step of bf16 each, and what fp32 sums differ by); strided inputs are
    taken."""
    G = matrices(shape, dtype, 8)
    O = b4.orth(G)
    turned = b4.orth(G.transpose(-1, -2)).transpose(-1, -2)
    if dtype == F32 or min(shape[-2:]) > 80:
        assert torch.equal(turned, O)
    else:
        assert ((turned.float() - O.float()).abs() <= 2 * 2.0 ** -8 * O.float().abs() + 1e-5).all()
    wide = torch.zeros(*shape[:-1], 2 * shape[-1], dtype=dtype, device="cuda")
    wide[..., ::2] = G
    assert torch.equal(b4.orth(wide[..., ::2]), O)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(5, 24, 100), (5, 100, 24), (5, 140, 100)], ids=str)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_bad_matrices_alone(shape, dtype, bad):
    G = matrices(shape, dtype, 9)
    O = b4.orth(G)
    G[0, 0, 0] = G[3, -1, -1] = bad
    got = b4.orth(G)
    assert got[[0, 3]].isnan().all() and torch.equal(got[[1, 2, 4]], O[[1, 2, 4]])


def test_batches():
    """A batch is its matrices one by one, also where the workspace takes a part of it at a time: the same
    bits in one batch wherever a matrix stands, and within the bound of what it is alone (the number of
    matrices may choose other tiles, and other orders of sums)."""
    for shape in ((37, 33, 100), (3, 140, 200), (2, 300, 900)):
        G = matrices(shape, F32, 10)
        G[-1] = G[0]
        O = b4.orth(G)
        assert torch.equal(O[-1], O[0])
        ref, bound = orth_ref(G)
        for k in (0, 1):
            close(b4.orth(G[k]), ref[k:k + 1], bound[k:k + 1], f"{shape} alone")
    G = matrices((6000, 96, 100), F32, 11, "spread")
    assert b4.lib().birkhoff4_orth_work(6000, 96, 100, b4.F32) <= 1 << 30
    G[1500] = G[5999] = G[3500].clone()
    O = b4.orth(G)
    ref, bound = orth_ref(G[[0, 1500]])
    close(O[[0, 1500]], ref, bound, "6000 matrices")
    assert torch.equal(O[1500], O[3500])
    close(O[5999:], ref[1:], bound[1:], "the last part")
    assert b4.orth(G[:0]).shape == (0, 96, 100) and b4.orth(G[:, :0]).shape == (6000, 0, 100)


@pytest.mark.parametrize("rows,cols", [(128, 1000), (24, 8200), (8200, 24)])
def test_far_matrices(rows, cols):
    """Batches beyond 2^31 values and 2^32 bytes: the last matrix, which is the first one again, has its bits."""
    B = (1 << 31) // (rows * cols) + 300
    G = torch.empty(B, rows, cols, dtype=BF16, device="cuda")
    for k in range(0, B, 2000):
        G[k:k + 2000] = matrices((rows, cols), BF16, k, "spread")
    G[-1] = G[0]
    O = b4.orth(G)
    assert torch.equal(O[-1], O[0]) and not torch.equal(O[-1], O[-2])
    ref, bound = orth_ref(G[:1], split=False)
    close(O[-1:], ref, bound, "last")
    if rows == 24:
        M, W = torch.zeros(B, rows, cols, device="cuda"), torch.ones(B, rows, cols, dtype=BF16, device="cuda")
        b4.orth_step(W, G, M, 0.1)
        assert torch.equal(W[-1], W[0]) and torch.equal(M[-1], G[0].float()) and not torch.equal(W[-1], W[-2])


@pytest.mark.parametrize("shape,dtype", [((3, 17, 45), F32), ((2, 150, 131), BF16), ((131, 150), F32)], ids=str)
def test_nothing_behind(shape, dtype):
    G = matrices(shape, dtype, 12)
    whole = torch.full((G.numel() + 130,), -7.0, dtype=dtype, device="cuda")
    out = whole[65:65 + G.numel()]  # beginning at any value
    lib, code = b4.lib(), b4.F32 if dtype == F32 else b4.BF16
    B, rows, cols = G.numel() // (shape[-1] * shape[-2]), *shape[-2:]
    size = lib.birkhoff4_orth_work(B, rows, cols, code)
    room = torch.full((size + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    array, steps = b4._steps(b4.ORTH_COEFS, 5)
    assert lib.birkhoff4_orth(G.data_ptr(), code, out.data_ptr(), code, array, steps, 1e-7, room[256:].data_ptr(), size, B, rows,
                              cols, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(out.view(G.shape), b4.orth(G))
    assert (whole[:65] == -7).all() and (whole[65 + G.numel():] == -7).all()
    assert (room[:256] == 0x5A).all() and (room[256 + size:] == 0x5A).all()


def step_ref(W, G, M, lr, momentum, nesterov, decay, scale, split):
    """(W, M) in float64, and the bound of W's error per matrix but for its own rounding."""
    M1 = (M.double() * momentum + G.double())
    M32 = torch.addcmul(G.float(), M, torch.tensor(momentum, dtype=F32, device="cuda"))
    U = G.float() + momentum * M32 if nesterov else M32
    O, bound = orth_ref(U, split=split)
    O = O.reshape(W.shape)
    if scale is None:
        scale = math.sqrt(max(1.0, W.shape[-2] / W.shape[-1]))
    ref = (1 - lr * decay) * W.double() - lr * scale * O
    # an fma, and lr, decay and scale as fp32 numbers: four roundings of each term
    slack = 4 * 2.0 ** -24 * (torch.linalg.vector_norm(W.double().reshape(O.shape), dim=(-2, -1)) + lr * scale * O.norm(dim=(-2, -1)))
    return ref, M1, bound * lr * scale * 1.001 + slack.reshape(bound.shape)


STEPS = [((24, 600), F32, F32), ((2, 80, 333), F32, BF16), ((150, 333), BF16, F32), ((2, 333, 150), BF16, BF16), ((65, 200), F32, BF16),
         ((1, 1), F32, F32), ((300, 20), BF16, F32)]


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shape,w_dtype,g_dtype", STEPS, ids=str)
def test_step(shape, w_dtype, g_dtype, nesterov):
    W, G, M = matrices(shape, w_dtype, 13, "spread", 0.1), matrices(shape, g_dtype, 14), matrices(shape, F32, 15)
    for lr, momentum, decay, scale in ((0.02, 0.95, 0.1, None), (0.5, 0.0, 0.0, 0.2), (0.0, 0.9, 0.5, 1.0)):
        ref, M1, bound = step_ref(W, G, M, lr, momentum, nesterov, decay, scale, w_dtype == F32)
        w, m = W.clone(), M.clone()
        versions = w._version, m._version
        assert b4.orth_step(w, G, m, lr, momentum, nesterov, decay, scale) is None
        assert w._version > versions[0] and m._version > versions[1]
        close(w, ref.reshape(-1, *shape[-2:]), bound, f"{shape} {w_dtype} {g_dtype} W")
        # one fma
        assert ((m.double() - M1).abs() <= 2.0 ** -24 * M1.abs() + 2.0 ** -23 * momentum * M.double().abs() + 1e-37).all()
        # the rate from the device
        w2, m2 = W.clone(), M.clone()
        b4.orth_step(w2, G, m2, torch.tensor(lr, device="cuda"), momentum, nesterov, decay, scale)
        assert torch.equal(w2, w) and torch.equal(m2, m)


@pytest.mark.parametrize("steps", [2, 3, 4, 5, 7])
@pytest.mark.parametrize("kind", ["mixed", "spread"])
def test_step_without_x(steps, kind):
    """Rectangular fp32 weights, whose steps run on the smaller side's products alone: the direction itself, read off
    weights of zero. It may be off by 1.6 times what the direct steps are, whose bound has a factor of three."""
    for shape in ((1280, 6000), (6000, 1280), (2, 1300, 5200)):
        G, M = matrices(shape, F32, 40 + steps, kind), torch.zeros(shape, device="cuda")
        W = torch.zeros(shape, device="cuda")
        b4.orth_step(W, G, M, -1.0, momentum=0.0, scale=1.0, steps=steps)
        ref, bound = orth_ref(G, steps=steps)
        close(W, ref, 1.6 * bound, f"{shape} {steps} {kind}")


def test_step_growing():
    """Steps without X whose coefficients are large away from zero, not at it."""
    shape, coefs = (1280, 6000), ((1.0, 1600.0, 0.0), (1.0, 10.0, 0.0), (1.5, -0.5, 0.0))
    G, M, W = matrices(shape, F32, 12, "spread"), torch.zeros(shape, device="cuda"), torch.zeros(shape, device="cuda")
    b4.orth_step(W, G, M, -1.0, momentum=0.0, scale=1.0, steps=3, coefs=coefs)
    ref, bound = orth_ref(G, steps=3, coefs=coefs)
    close(W, ref, 1.6 * bound, "growing")


def test_step_groups():
    """More matrices than the workspace takes at a time, with the steps without X: each as by itself."""
    shape = (9, 1280, 6000)
    assert b4.lib().birkhoff4_orth_work(*shape, b4.F32) < b4.lib().birkhoff4_orth_work(1, *shape[1:], b4.F32) * 9
    G, M, W = matrices(shape, BF16, 50), torch.zeros(shape, device="cuda"), torch.zeros(shape, device="cuda")
    G[-1] = G[0]
    b4.orth_step(W, G, M, -1.0, momentum=0.0, scale=1.0)
    ref, bound = orth_ref(G[[0, 5]].float())
    close(W[[0, 5]], ref, 1.6 * bound, "first and sixth")
    close(W[8:], ref[:1], 1.6 * bound[:1], "last")


def test_step_pieces():
    """Weights and momenta that begin at any value of a flat buffer; strided gradients."""
    shape = (45, 131)
    n = 45 * 131
    W, G, M = matrices(shape, F32, 16), matrices(shape, BF16, 17), matrices(shape, F32, 18)
    flat = torch.full((2 * n + 3,), -7.0, device="cuda")
    w, m = flat[1:1 + n].view(shape), flat[n + 2:2 * n + 2].view(shape)
    w.copy_(W)
    m.copy_(M)
    b4.orth_step(W, G, M, 0.1)
    b4.orth_step(w, G.t().contiguous().t(), m, 0.1)
    assert torch.equal(w, W) and torch.equal(m, M)
    assert flat[0] == -7 and flat[n + 1] == -7 and flat[-1] == -7


def test_refusals():
    W, G, M = (matrices((30, 20), F32, 19 + k) for k in range(3))
    for bad, error in (((G.half(),), TypeError), ((G[0],), ValueError), ((G.cpu(),), b4.Birkhoff4Error), ((G, 0), ValueError),
                       ((G, 5, (1.0, 2.0)), ValueError), ((G, 5, b4.ORTH_COEFS, -1.0), b4.Birkhoff4Error)):
        with pytest.raises(error):
            b4.orth(*bad)
    for bad, error in (((W, G[:, :19], M, 0.1), ValueError), ((W, G, M.bfloat16(), 0.1), TypeError), ((W.t(), G.t(), M.t(), 0.1), ValueError),
                       ((W, G.half(), M, 0.1), TypeError), ((W, G.cpu(), M, 0.1), b4.Birkhoff4Error), ((W, G, M[:29], 0.1), ValueError),
                       ((W, W, M, 0.1), b4.Birkhoff4Error), ((W, G, W, 0.1), b4.Birkhoff4Error),
                       ((W, G, M, torch.tensor(0.1)), b4.Birkhoff4Error), ((W, G, M, torch.ones(2, device="cuda")), ValueError),
                       ((W, G, M, torch.tensor(0.1, dtype=torch.float64, device="cuda")), TypeError)):
        with pytest.raises(error):
            b4.orth_step(*bad)
    P = W.clone().requires_grad_(True)
    with pytest.raises(RuntimeError, match="no derivative"):
        b4.orth_step(P, G, M, 0.1)
    with torch.no_grad():
        b4.orth_step(P, G, M, 0.1)
    with pytest.raises(RuntimeError, match="no derivative"):
        b4.orth_step(W, G, M, torch.tensor(0.1, device="cuda", requires_grad=True))


@pytest.mark.parametrize("shape,dtype", [((24, 500), F32), ((2, 200, 140), BF16)], ids=str)
def test_graphs(shape, dtype):
    """Two captured updates, replayed between eager work with the rate changed on the device, give the
    eager bits step after step."""
    W, M = matrices(shape, dtype, 20, "spread", 0.1), matrices(shape, F32, 21)
    G = [matrices(shape, BF16, 22 + k) for k in range(4)]
    eager = [(W.clone(), M.clone()) for _ in range(2)]
    held = [(W.clone(), M.clone(), G[0].clone(), torch.tensor(0.1, device="cuda")) for _ in range(2)]
    spare = W.clone(), M.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b4.orth_step(spare[0], G[0], spare[1], 0.1)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, (w, m, grad, lr) in zip(graphs, held):
        with torch.cuda.graph(g):
            b4.orth_step(w, grad, m, lr, decay=0.1)
    for turn in range(4):
        rate = 0.1 / (turn + 1)
        for k in range(2):
            held[k][2].copy_(G[(turn + k) % 4])
            held[k][3].fill_(rate)
            b4.orth_step(eager[k][0], G[(turn + k) % 4], eager[k][1], torch.tensor(rate, device="cuda"), decay=0.1)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (w, m, _, _), (we, me) in zip(held, eager):
            assert torch.equal(w, we) and torch.equal(m, me)


def test_other_stream():
    G = matrices((2, 300, 200), F32, 30)
    O = b4.orth(G)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = b4.orth(G)
    side.synchronize()
    assert torch.equal(O, again)


@pytest.mark.parametrize("n", [4, 8])
def test_training_step(n):
    """A step of a layer: connect with a norm in front of its branch, gradients, and the update of the
    coefficients' matrix and the branch's weights, against the same in float64 from the gradients."""
    g = torch.Generator(device="cuda").manual_seed(31)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)
    B, C, R = 60, 64, n * n + 2 * n
    X, T = normal(B, n, C), normal(B, n, C)
    W = torch.nn.Parameter(normal(R, n * C) / math.sqrt(n * C))
    V = torch.nn.Parameter(normal(C, C) / math.sqrt(C))
    rest = [torch.nn.Parameter(t) for t in (torch.ones(3, device="cuda"), torch.zeros(R, device="cuda"), torch.ones(C, device="cuda"),
                                            torch.zeros(C, device="cuda"))]
    M = [torch.zeros_like(W), torch.zeros_like(V)]
    for turn in range(3):
        Y = b4.connect(X, W, rest[0], rest[1], lambda U: torch.tanh(U @ V), norm=(rest[2], rest[3]))
        grads = torch.autograd.grad(((Y - T) ** 2).mean(), [W, V, *rest])
        assert all(x.isfinite().all() and x.abs().max() > 0 for x in grads)
        with torch.no_grad():
            for p, grad, m in zip((W, V), grads, M):
                ref, M1, bound = step_ref(p.detach().clone(), grad, m.clone(), 0.02, 0.95, True, 0.1, None, True)
                b4.orth_step(p, grad, m, 0.02, decay=0.1)
                close(p.detach(), ref.reshape(-1, *p.shape), bound, f"step {turn}")
            for p, grad in zip(rest, grads[2:]):
                p -= 0.01 * grad
