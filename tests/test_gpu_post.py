"""GPU parity of the streams' write (birkhoff*_post_fwd / _post_bwd) and of a whole layer (connect).

P is held to be what the projection alone gives, bit for bit; Y and the gradients are compared with
float64 on that P within the bounds of tests/_streams.py, and dH with the oracle's derivative by the
projection backward's own bound."""
import numpy as np
import pytest
import torch

import paper_2606_07574_amd as b4
from oracle import bwd as o_bwd4
from oracle import birkhoffn
from tests._gpu import TOL_DH
from tests._streams import kept, post_ref, within

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
SEED, OFFSET = 0x0123456789ABCDEF, (5 << 32) + 7


def inputs(n, B, C, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)
    H = normal(B, n, n) + 2 * torch.eye(n, device="cuda")
    return H, normal(B, n, C).to(dtype), 2 * torch.rand(B, n, device="cuda", generator=g), normal(B, C).to(dtype), \
        normal(B, n, C).to(dtype)


def words(seed=SEED, offset=OFFSET):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def check(H, X, h, Z, dY, p, label, keep=None):
    n = H.shape[-1]
    print(label, flush=True)
    if keep is None:
        keep = kept(Z.shape, p, SEED, OFFSET) if p else torch.ones(Z.shape, dtype=torch.bool)
    rng = words() if p else None
    Y, P, dual, it = b4.post_fwd(H, X, h, Z, p, rng, want_dual=True, want_iters=True)
    dX, dH, dh, dZ = b4.post_bwd(P, X, h, Z, dY, p, rng)
    alone = (b4.fwd if n == 4 else b4.fwd8)(H, want_iters=True)
    torch.cuda.synchronize()
    for a, b in zip((P, dual, it), alone):
        assert torch.equal(a, b), label
    within(Y, *post_ref(P, X, h, Z, keep, p), "Y")
    ref, err = post_ref(P, X, h, Z, keep, p, dY)
    within(dX, ref[0], err[0], "dX")
    within(dh, ref[2], err[2], "dh")
    within(dZ, ref[3], err[3], "dZ")
    assert (dZ[~keep.cuda()] == 0).all()
    dHr = (o_bwd4 if n == 4 else birkhoffn.bwd)(P.cpu().numpy().astype(np.float64), ref[1].cpu().numpy())
    d = np.abs(dH.cpu().numpy() - dHr).reshape(len(dHr), -1).max(1) / np.maximum(1, np.abs(dHr).reshape(len(dHr), -1).max(1))
    assert not len(d) or d.max() <= TOL_DH, f"{label}: dH {d.max()}"


# one token of every row length's kernel; few tokens (one launch) and many; rows of 1 to 8 chunks,
# 9 to 16, 17 to 32, one, two and several columns of 64, whole and ragged
SIZES = [(1, 8), (1, 4096), (3, 64), (9, 72), (33, 128), (5, 136), (70, 256), (31, 264), (40, 520), (17, 1032),
         (2500, 8), (2300, 136), (2200, 520), (300, 4104)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [4, 8])
@pytest.mark.parametrize("B,C", SIZES)
def test_sizes(n, B, C, dtype):
    C = C if dtype == BF16 else C // 2
    p = (0.0, 0.1, 0.5)[(B + C) % 3] if B * C < 400000 else 0.0
    check(*inputs(n, B, C, dtype, 10 * n + B), p, f"n={n} B={B} C={C} {dtype} p={p}")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [4, 8])
@pytest.mark.parametrize("p", [2.0 ** -33, 1e-3, 0.9, 0.999])
def test_probabilities(n, p, dtype):
    """Down to one that never drops (floor(p 2^32) = 0) and up to one that leaves whole tokens
    without an element."""
    check(*inputs(n, 60, 40, dtype, 3), p, f"n={n} p={p}")


def test_mask_alone():
    """The mask depends on the element's index, p and rng alone: not on the dtype, the number of
    streams or the kernel; and another seed or offset gives another."""
    B, C, p = 200, 1032, 0.3
    masks = []
    for n, dtype in ((4, F32), (4, BF16), (8, F32), (8, BF16)):
        H, X, h, Z, dY = inputs(n, B, C, dtype, 5)
        Y = b4.post_fwd(H, torch.zeros_like(X), torch.ones_like(h), torch.ones_like(Z), p, words())[0]
        masks.append(Y[:, 0] != 0)
        assert (Y[:, :1] == Y).all()
    for m in masks:
        assert torch.equal(m, masks[0])
    assert torch.equal(masks[0].cpu(), kept((B, C), p, SEED, OFFSET))
    H, X, h, Z, _ = inputs(4, B, C, F32, 5)
    for other in (words(SEED + 1), words(SEED, OFFSET + 1), words(SEED + (1 << 40)), words(SEED, OFFSET + (1 << 40)),
                  words(-1, -1)):
        Y = b4.post_fwd(H, torch.zeros_like(X), torch.ones_like(h), torch.ones_like(Z), p, other)[0]
        # two independent masks agree in p^2 + (1 - p)^2 = 0.58 of the elements, sigma 0.0011
        assert abs((masks[0] == (Y[:, 0] != 0)).float().mean().item() - 0.58) < 0.006
        # and keep 0.7 of them, sigma 0.0010
        assert abs((Y[:, 0] != 0).float().mean().item() - 0.7) < 0.006
    assert torch.equal((Y[:, 0] != 0).cpu(), kept((B, C), p, -1, -1))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 3e38])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_masked_values(dtype, bad):
    """What is dropped does not count, whatever it holds."""
    H, X, h, Z, dY = inputs(4, 50, 72, dtype, 7)
    keep = kept(Z.shape, 0.5, SEED, OFFSET)
    Z[~keep.cuda()] = bad
    check(H, X, h, Z, dY, 0.5, f"masked {bad}", keep)


def test_no_tokens_no_channels():
    for n in (4, 8):
        H, X, h, Z, dY = inputs(n, 0, 64, BF16, 9)
        Y, P, _, _ = b4.post_fwd(H, X, h, Z, 0.1, words())
        assert Y.shape == X.shape
        assert all(t.numel() == 0 for t in b4.post_bwd(P, X, h, Z, dY, 0.1, words()))
        H, X, h, Z, dY = inputs(n, 5, 0, F32, 9)
        Y, P, _, _ = b4.post_fwd(H, X, h, Z)
        dX, dH, dh, dZ = b4.post_bwd(P, X, h, Z, dY)
        assert Y.numel() == 0 and torch.equal(P, (b4.fwd if n == 4 else b4.fwd8)(H)[0])
        assert (dh == 0).all() and (dH == 0).all()


def test_same_as_mix():
    """With h = 0 it is the residual mixing: the same P, and the same streams up to fp32's order."""
    for n in (4, 8):
        H, X, h, Z, dY = inputs(n, 500, 264, F32, 11)
        Y, P, _, _ = b4.post_fwd(H, X, torch.zeros_like(h), Z)
        Ym, Pm, _, _ = (b4.mix_fwd if n == 4 else b4.mix8_fwd)(H, X)
        assert torch.equal(P, Pm) and (Y - Ym).abs().max() <= 2 * n * 2.0 ** -24 * X.abs().sum(1).max()
        dX, dH, _, _ = b4.post_bwd(P, X, torch.zeros_like(h), Z, dY)
        dXm, dHm = (b4.mix_bwd if n == 4 else b4.mix8_bwd)(P, X, dY)
        assert torch.equal(dX, dXm) and torch.equal(dH, dHm)


@pytest.mark.parametrize("n,h_dtype,dtype", [(4, F32, BF16), (4, BF16, BF16), (8, BF16, BF16), (8, F32, F32)])
def test_autograd(n, h_dtype, dtype):
    """post under autograd, with leading dimensions and strides: the same as the pair of calls."""
    H, X, h, Z, dY = inputs(n, 12, 264, dtype, 13)
    H = H.to(h_dtype)
    lead = lambda t: t.reshape(3, 4, *t.shape[1:])
    args = [lead(H), lead(X).transpose(0, 1).contiguous().transpose(0, 1), lead(h), lead(Z)]
    args = [a.detach().requires_grad_() for a in args]
    rng = words()
    Y = b4.post(*args, 0.1, rng)
    got = torch.autograd.grad(Y, args, lead(dY))
    Yr, P, _, _ = b4.post_fwd(H, X, h, Z, 0.1, rng)
    dX, dH, dh, dZ = b4.post_bwd(P, X, h, Z, dY, 0.1, rng)
    assert torch.equal(Y.detach().reshape(Yr.shape), Yr)
    for a, b in zip(got, (dH.to(h_dtype), dX, dh, dZ)):
        assert a.dtype == b.dtype and torch.equal(a.reshape(b.shape), b)
    Y = b4.post(*args, 0.1, rng)
    rng[1] += 1  # the backward would draw another mask
    with pytest.raises(RuntimeError):
        Y.sum().backward()


def test_differences():
    """The gradient against central differences of the forward along random directions, fp32 (the
    steps and bounds of test_gpu_pre.py's; P stops within 1e-6 of the projection, 2^-14 of a step)."""
    H, X, h, Z, dY = inputs(4, 10, 32, F32, 15)
    args = [t.requires_grad_() for t in (H, X, h, Z)]
    rng = words()
    got = torch.autograd.grad(b4.post(*args, 0.25, rng), args, dY)
    plain = [a.detach() for a in args]
    g = torch.Generator(device="cuda").manual_seed(17)
    value = lambda vals: (b4.post_fwd(*vals, 0.25, rng)[0].double() * dY.double()).sum()
    step = 2.0 ** -6
    for k, name in enumerate("HXhZ"):
        D = torch.randn(plain[k].shape, device="cuda", generator=g)
        D /= D.norm()
        up, down = (plain[:k] + [plain[k] + s * D] + plain[k + 1:] for s in (step, -step))
        diff = ((value(up) - value(down)) / (2 * step)).item()
        size = (got[k].double() * D).abs().sum().item()
        assert abs(diff - (got[k].double() * D).sum().item()) <= 2.0 ** -10 * (size + got[k].norm().item()), name


def test_graph_draws_anew():
    """Captured with the generator's words advanced in the graph: each replay has the mask of the
    words it finds, and equals the eager calls with them."""
    H, X, h, Z, dY = inputs(4, 300, 264, BF16, 19)
    rng = words()

    def step(H, X, h, Z, dY, rng):
        rng[1] += 1
        Y, P, _, _ = b4.post_fwd(H, X, h, Z, 0.2, rng)
        return (Y, P, *b4.post_bwd(P, X, h, Z, dY, 0.2, rng))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(H, X, h, Z, dY, rng)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(H, X, h, Z, dY, rng)
    rng.copy_(words())
    before = None
    for k in range(3):
        for o in outs:
            o.fill_(float("nan"))
        graph.replay()
        ref = step(H, X, h, Z, dY, words(SEED, OFFSET + k))
        torch.cuda.synchronize()
        assert rng.tolist() == [SEED, OFFSET + k + 1]
        for a, b in zip(outs, ref):
            assert torch.equal(a, b)
        assert before is None or not torch.equal(before, outs[0])
        before = outs[0].clone()


def test_refusals():
    H, X, h, Z, dY = inputs(4, 10, 64, BF16, 21)
    P = b4.post_fwd(H, X, h, Z)[1]
    for p in (1.0, -0.1, 2.0, float("nan")):
        with pytest.raises(b4.Birkhoff4Error):
            b4.post_fwd(H, X, h, Z, p, words())
        with pytest.raises(b4.Birkhoff4Error):
            b4.post_bwd(P, X, h, Z, dY, p, words())
    bad = [(ValueError, dict(p=0.1)), (TypeError, dict(p=0.1, rng=words().int())), (ValueError, dict(p=0.1, rng=words()[:1])),
           (b4.Birkhoff4Error, dict(p=0.1, rng=words().cpu())), (TypeError, dict(h=h.bfloat16())), (TypeError, dict(Z=Z.float())),
           (ValueError, dict(h=h[:, :3].contiguous())), (ValueError, dict(Z=Z[:5])), (ValueError, dict(Z=Z.t().contiguous().t())),
           (b4.Birkhoff4Error, dict(Z=Z.cpu())), (ValueError, dict(X=X[:5]))]
    for error, kw in bad:
        with pytest.raises(error):
            b4.post_fwd(**{**dict(H=H, X=X, h=h, Z=Z), **kw})
        with pytest.raises(error):
            b4.post_bwd(**{**dict(P=P, X=X, h=h, Z=Z, dY=dY), **kw})
    with pytest.raises(ValueError):
        b4.post_fwd(H[:, :3, :3].contiguous(), X, h, Z)
    with pytest.raises(TypeError):
        b4.post_bwd(P.bfloat16(), X, h, Z, dY)


# ---------------------------------------------------------------------------
# Whole layers
# ---------------------------------------------------------------------------
def layer64(X, W, alpha, bias, branch, eps, keep, p):
    """One layer in float64 under autograd, its projection by 300 sweeps (unit-scale logits)."""
    n, C = X.shape[-2:]
    x = X.reshape(-1, n * C)
    a = torch.cat([alpha[:1].expand(n), alpha[1:2].expand(n), alpha[2:].expand(n * n)])
    l = a * ((x @ W.t()) * (x.square().mean(1, keepdim=True) + eps).rsqrt()) + bias
    U = (torch.sigmoid(l[:, :n, None]) * X).sum(1)
    P = torch.exp(l[:, 2 * n:].reshape(-1, n, n))
    for _ in range(300):
        P = P / P.sum(1, keepdim=True)
        P = P / P.sum(2, keepdim=True)
    D = branch(U) * (keep.to(X.device).double() / (1 - p))
    return P @ X + 2 * torch.sigmoid(l[:, n:2 * n, None]) * D[:, None]


@pytest.mark.parametrize("n,dtype,tol", [(4, F32, 1e-4), (8, F32, 1e-4), (4, BF16, 12 * 2.0 ** -8), (8, BF16, 12 * 2.0 ** -8)])
def test_two_layers(n, dtype, tol):
    """Two layers around a branch with weights of its own, forward and backward, against float64.
    fp32: P is within 1e-5 of the projection and its derivative within 1e-4 of the oracle's, in each
    layer. bf16: U, the branch's two products, Y and their gradients are rounded in each of two
    layers, twelve roundings of at most 2^-8 one after the other."""
    g = torch.Generator(device="cuda").manual_seed(23)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)
    B, C, p, eps = 45, 64, 0.25, 1e-6
    K, N = n * C, n * n + 2 * n
    eye = torch.cat([torch.zeros(2 * n, device="cuda"), 2 * torch.eye(n, device="cuda").flatten()])
    params, rngs, keeps = [], [], []
    for k in range(2):
        params.append([(normal(N, K) / K ** 0.5).to(dtype), 1 + 0.1 * normal(3), 0.5 * normal(N) + eye,
                       (normal(C, C) / C ** 0.5).to(dtype)])
        rngs.append(words(SEED, k))
        keeps.append(kept((B, C), p, SEED, k))
    X, dY = normal(B, n, C).to(dtype), normal(B, n, C).to(dtype)

    def run(cast, layer):
        leaves = [cast(X).requires_grad_()] + [cast(t).requires_grad_() for ps in params for t in ps]
        x = leaves[0]
        for k in range(2):
            W, alpha, bias, M = leaves[1 + 4 * k:5 + 4 * k]
            x = layer(k, x, W, alpha, bias, lambda U: torch.tanh(U @ M))
        return (x, *torch.autograd.grad(x, leaves, cast(dY)))

    got = run(lambda t: t.detach().clone(), lambda k, x, W, a, b, f: b4.connect(x, W, a, b, f, p, rngs[k], eps))
    ref = run(lambda t: t.detach().double(), lambda k, x, W, a, b, f: layer64(x, W, a, b, f, eps, keeps[k], p))
    for k, (a, b) in enumerate(zip(got, ref)):
        off = ((a.double() - b).norm() / b.norm()).item()
        print(f"  output {k}: {off:.2e}", flush=True)
        assert off <= tol, k


def test_connect_without_gradients():
    g = torch.Generator(device="cuda").manual_seed(25)
    X = torch.randn(7, 4, 64, device="cuda", generator=g)
    W = torch.randn(24, 256, device="cuda", generator=g) / 16
    alpha, bias = torch.ones(3, device="cuda"), torch.zeros(24, device="cuda")
    with torch.no_grad():
        Y = b4.connect(X, W, alpha, bias, torch.tanh)
    U, h, H, _, _ = b4.pre_fwd(X, W, alpha, bias)
    assert not Y.requires_grad and torch.equal(Y, b4.post_fwd(H, X, h, torch.tanh(U))[0])


@pytest.mark.parametrize("n", [4, 8])
def test_far_tokens(n):
    """Streams of more than 2^31 values: the last tokens' outputs, forward and backward."""
    C, last = 4096, 40
    B = (1 << 31) // (n * C) + 1000
    g = torch.Generator(device="cuda").manual_seed(27)
    X = torch.randn(B, n, C, device="cuda", generator=g, dtype=BF16)
    N, K = n * n + 2 * n, n * C
    W = (torch.randn(N, K, device="cuda", generator=g) / K ** 0.5).to(BF16)
    alpha, bias = torch.ones(3, device="cuda"), torch.randn(N, device="cuda", generator=g)
    U, h, H, q, rms = b4.pre_fwd(X, W, alpha, bias)
    from tests._streams import pre_back_ref, pre_ref
    cut = slice(B - last, B)
    out, err, ref = pre_ref(X[cut], W, alpha, bias, 1e-6)
    for k, t in zip(("U", "h", "H", "q", "rms"), (U, h, H, q, rms)):
        within(t[cut], out[k], err[k], k)
    Y, P, _, _ = b4.post_fwd(H, X, h, U)
    keep = torch.ones(last, C, dtype=torch.bool)
    within(Y[cut], *post_ref(P[cut], X[cut], h[cut], U[cut], keep, 0.0), "Y")
    dX, dH, dh, dZ = b4.post_bwd(P, X, h, U, Y)
    r, e = post_ref(P[cut], X[cut], h[cut], U[cut], keep, 0.0, Y[cut])
    within(dX[cut], r[0], e[0], "dX")
    within(dZ[cut], r[3], e[3], "dZ")
    del Y
    dX2 = b4.pre_bwd(X, W, alpha, bias, q, rms, dZ, dh, dH, dX)[0]
    (r, *_), (e, *_) = pre_back_ref(ref, n, dZ[cut], dh[cut], dH[cut], dX[cut])
    within(dX2[cut], r, e, "dX of pre")


def test_no_second_derivatives():
    """A gradient taken with create_graph is right, and its own derivative is refused, not taken as zero."""
    g = torch.Generator(device="cuda").manual_seed(27)
    X = torch.randn(5, 4, 64, device="cuda", generator=g, requires_grad=True)
    W = torch.randn(24, 256, device="cuda", generator=g) / 16
    alpha, bias = torch.ones(3, device="cuda"), torch.zeros(24, device="cuda")
    U, h, H, Xs = b4.pre(X, W, alpha, bias)
    for out in (U, b4.post(H.detach(), X, h.detach(), U.detach())):
        once, = torch.autograd.grad(out.square().sum(), X, create_graph=True, retain_graph=True)
        plain, = torch.autograd.grad(out.square().sum(), X, retain_graph=True)
        assert torch.equal(once, plain)
        with pytest.raises(RuntimeError, match="differentiable"):
            once.square().sum().backward()
