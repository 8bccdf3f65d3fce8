"""GPU parity of the streams' read (birkhoff*_pre_fwd / _pre_bwd) with float64, element by element,
within bounds that follow from the sums' magnitudes (tests/_streams.py)."""
import pytest
import torch

import paper_2606_07574_amd as b4
from tests._streams import pre_back_ref, pre_ref, within

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
DTYPES = [F32, BF16]


def inputs(n, B, C, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)
    K, N = n * C, n * n + 2 * n
    X = (scale * normal(B, n, C)).to(dtype)
    W = (normal(N, K) / K ** 0.5).to(dtype)
    alpha, bias = 1.0 + 0.2 * normal(3), normal(N)
    grads = normal(B, C).to(dtype), normal(B, n), normal(B, n, n), normal(B, n, C).to(dtype)
    return X, W, alpha, bias, grads


def check(X, W, alpha, bias, grads, eps, label):
    n = X.shape[-2]
    print(f"{label}", flush=True)
    got = dict(zip(("U", "h", "H", "q", "rms"), b4.pre_fwd(X, W, alpha, bias, eps)))
    back = b4.pre_bwd(X, W, alpha, bias, got["q"], got["rms"], *grads)
    torch.cuda.synchronize()
    out, err, ref = pre_ref(X, W, alpha, bias, eps)
    for k in out:
        within(got[k], out[k], err[k], k)
    for k, g, r, e in zip(("dX", "dW", "dalpha", "dbias"), back, *pre_back_ref(ref, n, *grads)):
        within(g, r, e, k)


# one token to several steps of 32 and tiles of 16, 32 and 64 with remainders; rows shorter than a
# lane group's chunk, of odd numbers of chunks, of several columns of 64 chunks
SIZES = [(1, 8), (1, 4096), (2, 40), (15, 24), (16, 264), (17, 8), (31, 136), (33, 520), (63, 72), (64, 1032),
         (65, 128), (257, 248), (1000, 16), (300, 2056)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [4, 8])
@pytest.mark.parametrize("B,C", SIZES)
def test_sizes(n, B, C, dtype):
    C = C if dtype == BF16 else C // 2
    check(*inputs(n, B, C, dtype, 100 * n + B), 1e-6, f"n={n} B={B} C={C} {dtype}")


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [4, 8])
def test_many_tokens(n, dtype):
    """More tokens than the backward's blocks take in one turn, and than one share has steps."""
    check(*inputs(n, 20011, 64, dtype, 7), 1e-6, f"n={n} many tokens {dtype}")


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n,B,C", [(4, 20481, 72), (4, 21000, 40), (8, 2049, 72), (8, 2500, 264), (8, 2304, 8)])
def test_blocks_of_many_tokens(n, B, C, dtype):
    """Waves with 64 tokens each that share W's lines: rows of odd numbers of 64-byte steps, blocks
    whose last waves have no tokens, shares of the row."""
    C = C if dtype == BF16 else C // 2
    check(*inputs(n, B, C, dtype, 43), 1e-6, f"n={n} B={B} C={C} {dtype}")


@pytest.mark.parametrize("scale,eps", [(1e-4, 1e-6), (1e-4, 0.0), (300.0, 1e-6), (1.0, 0.5)])
def test_scales(scale, eps):
    check(*inputs(4, 50, 256, F32, 3, scale), eps, f"scale {scale}, eps {eps}")
    check(*inputs(8, 50, 256, BF16, 3, scale), eps, f"scale {scale}, eps {eps}, bf16")


@pytest.mark.parametrize("given", [(1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (0, 0, 0, 0), (1, 1, 1, 0)])
def test_missing_gradients(given):
    """Gradients that are not there count as zeros."""
    X, W, alpha, bias, grads = inputs(4, 70, 136, BF16, 5)
    check(X, W, alpha, bias, [g if k else None for g, k in zip(grads, given)], 1e-6, f"gradients {given}")


def test_zero_streams():
    """|v| = 0: r = eps^(-1/2), every coefficient its bias's."""
    X, W, alpha, bias, grads = inputs(4, 40, 64, F32, 9)
    X.zero_()
    check(X, W, alpha, bias, grads, 1e-2, "zero streams")


@pytest.mark.parametrize("n", [4, 8])
def test_saturated_gates(n):
    """Biases far beyond where a sigmoid is 0 or 1 in fp32: the gates are exactly that, and pass
    no gradient."""
    X, W, alpha, bias, grads = inputs(n, 33, 64, F32, 11)
    bias[:n] = torch.where(torch.arange(n, device="cuda") % 2 == 0, 300.0, -300.0)
    bias[n:2 * n] = -bias[:n]
    U, h, H, q, rms = b4.pre_fwd(X, W, alpha, bias)
    assert torch.equal(h[:, 0::2], torch.zeros_like(h[:, 0::2])) and (h[:, 1::2] == 2).all()
    even = sum(X[:, i] for i in range(0, n, 2))
    assert (U - even).abs().max() <= 4 * 2.0 ** -24 * X.abs().sum(1).max()
    _, dW, _, dbias = b4.pre_bwd(X, W, alpha, bias, q, rms, *grads)
    assert (dbias[:2 * n] == 0).all() and (dW[:2 * n] == 0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n,dtype", [(4, BF16), (8, F32), (8, BF16), (4, F32)])
def test_non_finite_token(n, dtype, bad):
    """A token with a NaN or infinite value leaves every other token's outputs as they were."""
    X, W, alpha, bias, grads = inputs(n, 75, 72, dtype, 13)
    clean = b4.pre_fwd(X, W, alpha, bias)
    dclean = b4.pre_bwd(X, W, alpha, bias, clean[3], clean[4], *grads)[0]
    others = torch.arange(75, device="cuda") != 37
    X[37, n - 1, 5] = bad
    got = b4.pre_fwd(X, W, alpha, bias)
    dX, dW, dalpha, dbias = b4.pre_bwd(X, W, alpha, bias, got[3], got[4], *grads)
    for a, b in zip(got, clean):
        assert torch.equal(a[others], b[others])
    assert not torch.isfinite(got[0][37]).any()
    assert torch.equal(dX[others], dclean[others])
    assert not torch.isfinite(dW.float()).all() and not torch.isfinite(dbias).all()


def test_non_finite_last_token():
    """The tokens that pad the last step are not read for the products over tokens, whatever the
    last token holds."""
    X, W, alpha, bias, grads = inputs(4, 33, 64, BF16, 15)
    E = grads[3].clone()
    E[32] = float("nan")
    X2 = X.clone()
    q, rms = b4.pre_fwd(X2, W, alpha, bias)[3:]
    dX, dW, _, _ = b4.pre_bwd(X2, W, alpha, bias, q, rms, *grads[:3], E)
    assert dX[32].isnan().all() and torch.isfinite(dX[:32].float()).all() and torch.isfinite(dW.float()).all()


def test_deterministic():
    X, W, alpha, bias, grads = inputs(8, 3001, 200, BF16, 17)
    first = b4.pre_fwd(X, W, alpha, bias)
    second = b4.pre_fwd(X, W, alpha, bias)
    for a, b in zip(first, second):
        assert torch.equal(a, b)
    for a, b in zip(*(b4.pre_bwd(X, W, alpha, bias, first[3], first[4], *grads) for _ in range(2))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("n,dtype", [(4, BF16), (8, F32)])
def test_no_tokens(n, dtype):
    """Without tokens the sums over tokens are zeros."""
    X, W, alpha, bias, grads = inputs(n, 0, 64, dtype, 19)
    U, h, H, q, rms = b4.pre_fwd(X, W, alpha, bias)
    assert U.shape == (0, 64) and H.shape == (0, n, n)
    dX, dW, dalpha, dbias = b4.pre_bwd(X, W, alpha, bias, q, rms, *grads)
    assert dX.shape == X.shape
    for t in (dW, dalpha, dbias):
        assert (t == 0).all()


def test_neighbours_untouched():
    """Outputs of the C call end where they should: guard values behind them stay."""
    n, B, C = 4, 37, 40
    X, W, alpha, bias, _ = inputs(n, B, C, BF16, 21)
    N = n * n + 2 * n

    def guarded(numel, dtype):
        return torch.full((numel + 64,), 7.0, dtype=dtype, device="cuda")

    U, h, H, q, rms = (guarded(B * C, BF16), guarded(B * n, F32), guarded(B * n * n, F32), guarded(B * N, F32),
                       guarded(B, F32))
    size = b4.lib().birkhoff4_pre_work(B, C, b4.BF16, 0)
    work = torch.full((size + 64,), 7, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    code = b4.lib().birkhoff4_pre_fwd(X.data_ptr(), W.data_ptr(), b4.BF16, alpha.data_ptr(), bias.data_ptr(), 1e-6,
                                      U.data_ptr(), h.data_ptr(), H.data_ptr(), q.data_ptr(), rms.data_ptr(),
                                      work.data_ptr(), size, B, C, stream)
    assert code == 0
    ref = b4.pre_fwd(X, W, alpha, bias)
    for a, b in zip((U, h, H, q, rms), ref):
        assert torch.equal(a[:b.numel()], b.flatten()) and (a[b.numel():] == 7).all()
    assert (work[size:] == 7).all()


def grad_inputs(n, lead, C, dtype, seed):
    B = 1
    for k in lead:
        B *= k
    X, W, alpha, bias, grads = inputs(n, B, C, dtype, seed)
    shape = lambda t: t.reshape(*lead, *t.shape[1:])
    return [t.requires_grad_() for t in (shape(X), W, alpha, bias)], [shape(g) for g in grads]


@pytest.mark.parametrize("n,dtype", [(4, BF16), (8, F32)])
def test_autograd(n, dtype):
    """pre under autograd, with leading dimensions: the same as the pair of calls."""
    args, grads = grad_inputs(n, (3, 5), 96, dtype, 23)
    outs = b4.pre(*args)
    assert outs[3].data_ptr() == args[0].data_ptr()  # the streams themselves
    got = torch.autograd.grad(outs, args, grads)
    plain = [a.detach() for a in args]
    fwd = b4.pre_fwd(*plain)
    for a, b in zip(outs[:3], fwd):
        assert torch.equal(a.detach(), b)
    for a, b in zip(got, b4.pre_bwd(*plain, *fwd[3:], *grads)):
        assert torch.equal(a, b)
    # one output alone, and the streams' gradient alone
    outs = b4.pre(*args)
    (dW,) = torch.autograd.grad(outs[1], args[1], grads[1], retain_graph=True)
    assert torch.equal(dW, b4.pre_bwd(*plain, *fwd[3:], None, grads[1], None)[1])
    (dX,) = torch.autograd.grad(outs[3], args[0], grads[3])
    assert torch.equal(dX, grads[3])


def test_strided_inputs():
    """Under autograd a transposed or sliced X, W, bias or gradient is taken as the values it has."""
    (X, W, alpha, bias), grads = grad_inputs(4, (20,), 64, F32, 25)
    base = b4.pre(X, W, alpha, bias)
    ref = torch.autograd.grad(base, (X, W, alpha, bias), grads)
    Xs = X.detach().permute(1, 0, 2).contiguous().permute(1, 0, 2).requires_grad_()
    Ws = W.detach().t().contiguous().t().requires_grad_()
    bs = torch.stack([bias.detach(), bias.detach()], 1)[:, 0].requires_grad_()
    outs = b4.pre(Xs, Ws, alpha, bs)
    gs = [g.transpose(0, -1).contiguous().transpose(0, -1) for g in grads]
    for a, b in zip(torch.autograd.grad(outs, (Xs, Ws, alpha, bs), gs), ref):
        assert torch.equal(a, b)


def test_flat_parameters():
    """Parameters that are pieces of one flat buffer, off the kernels' 16 bytes, under autograd; the
    calls without it refuse them."""
    (X, W, alpha, bias), grads = grad_inputs(4, (20,), 64, F32, 45)
    ref = torch.autograd.grad(b4.pre(X, W, alpha, bias), (X, W, alpha, bias), grads)
    flat = torch.cat([t.detach().flatten() for t in (alpha, bias, W)]).requires_grad_()
    a, b, w = flat[:3], flat[3:27], flat[27:].view(24, 256)
    outs = b4.pre(X, w, a, b)
    got = torch.autograd.grad(outs, (X, flat), grads)
    assert torch.equal(got[0], ref[0])
    assert torch.equal(got[1], torch.cat([ref[2], ref[3], ref[1].flatten()]))
    with torch.no_grad():
        for x, y in zip(b4.pre(X, w, a, b), outs):
            assert torch.equal(x, y)
        with pytest.raises(b4.Birkhoff4Error, match="aligned"):
            b4.pre_fwd(X, W, a, b)


@pytest.mark.parametrize("n", [4, 8])
def test_differences(n):
    """The gradient against central differences of the forward along random directions, fp32. The
    function has second and third derivatives of the order of one per unit step, so at a step of
    2^-6 the difference's own error is about 2^-12 of the directional sums' size; rounding of the
    outputs (2^-22 of them) over the step adds 2^-16."""
    args, grads = grad_inputs(n, (12,), 32, F32, 27)
    got = torch.autograd.grad(b4.pre(*args), args, grads)
    plain = [a.detach() for a in args]
    g = torch.Generator(device="cuda").manual_seed(29)

    def value(vals):
        outs = (*b4.pre_fwd(*vals)[:3], vals[0])
        return sum((o.double() * k.double()).sum() for o, k in zip(outs, grads))

    step = 2.0 ** -6
    for k, name in enumerate(("X", "W", "alpha", "bias")):
        D = torch.randn(plain[k].shape, device="cuda", generator=g)
        D /= D.norm()  # unit length: the outputs move by at most about the step
        up, down = (plain[:k] + [plain[k] + s * D] + plain[k + 1:] for s in (step, -step))
        diff = ((value(up) - value(down)) / (2 * step)).item()
        size = (got[k].double() * D).abs().sum().item()
        assert abs(diff - (got[k].double() * D).sum().item()) <= 2.0 ** -10 * (size + got[k].norm().item()), name


def test_graph_and_streams():
    """Captured and replayed with new inputs, and run on another stream: the eager call's bits."""
    sets = [inputs(4, 200, 264, BF16, 31 + k) for k in range(3)]

    def both(X, W, alpha, bias, grads):
        f = b4.pre_fwd(X, W, alpha, bias)
        return (*f, *b4.pre_bwd(X, W, alpha, bias, f[3], f[4], *grads))

    X, W, alpha, bias, grads = sets[0]
    static = [X.clone(), W.clone(), alpha.clone(), bias.clone(), [g.clone() for g in grads]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = both(*static)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, b in zip(on_side, both(*sets[0])):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = both(*static)
    for s in sets:
        for d, v in zip(static[:4], s[:4]):
            d.copy_(v)
        for d, v in zip(static[4], s[4]):
            d.copy_(v)
        ref = both(*s)
        torch.cuda.synchronize()
        for _ in range(2):
            for o in outs:
                o.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(outs, ref):
                assert torch.equal(a, b)


def test_refusals():
    X, W, alpha, bias, grads = inputs(4, 10, 64, BF16, 41)
    ok = b4.pre_fwd(X, W, alpha, bias)
    refused = [
        (TypeError, (X, W.float(), alpha, bias)), (TypeError, (X.half(), W.half(), alpha, bias)),
        (TypeError, (X, W, alpha.double(), bias)), (TypeError, (X, W, alpha, bias.bfloat16())),
        (ValueError, (X, W[:-1], alpha, bias)), (ValueError, (X, W, alpha[:2], bias)), (ValueError, (X, W, alpha, bias[1:])),
        (ValueError, (X.transpose(0, 1), W, alpha, bias)), (ValueError, (X[:, :3].contiguous(), W, alpha, bias)),
        (ValueError, (X, W.t().contiguous().t(), alpha, bias)), (b4.Birkhoff4Error, (X.cpu(), W, alpha, bias)),
        (b4.Birkhoff4Error, (X, W.cpu(), alpha, bias)), (b4.Birkhoff4Error, (X, W, alpha, bias, -1.0)),
        (b4.Birkhoff4Error, (X, W, alpha, bias, float("nan"))), (b4.Birkhoff4Error, (X, W, alpha, bias, float("inf"))),
    ]
    for error, args in refused:
        with pytest.raises(error):
            b4.pre_fwd(*args)
    with pytest.raises(b4.Birkhoff4Error):  # rows of 12 bf16 values are not whole 16-byte chunks
        b4.pre_fwd(*inputs(4, 3, 12, BF16, 1)[:4])
    with pytest.raises(b4.Birkhoff4Error):  # no channels: no norm
        b4.pre_fwd(*(t[..., :0].contiguous() if t.dim() > 1 else t for t in (X, W, alpha, bias)))
    for k, g in enumerate((grads[0].float(), grads[1][:, :3].contiguous(), grads[2].bfloat16(), grads[3][:5])):
        bad = list(grads)
        bad[k] = g
        with pytest.raises((TypeError, ValueError)):
            b4.pre_bwd(X, W, alpha, bias, ok[3], ok[4], *bad)
    with pytest.raises(ValueError):
        b4.pre_bwd(X, W, alpha, bias, ok[3][:5], ok[4], *grads)


def pieces(v):
    """fp32 values as three bf16 ones that add up to them: the upper eight bits of the significand,
    the next eight and the last eight, so that each is exact."""
    upper = lambda t: (t.view(torch.int32) & -65536).view(F32)
    hi = upper(v)
    mid = upper(v - hi)
    return hi, mid, v - hi - mid


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [4, 8])
def test_gradient_of_products_is_whole(n, dtype):
    """G, the gradient of the products, enters dX = G W and dW = G^T X with all the 24 bits of its
    fp32 values, also where the streams are bf16: with r = alpha = 1 and q = 0 it is dH, W = 1 (X = 1)
    makes the product dH itself, and what takes its upper 16 bits away leaves the last eight, of
    which every sum on the way is a whole fp32 value. One row of W a token, so that nothing else
    is added."""
    N, C, M = n * n + 2 * n, 72, n * n
    g = torch.Generator(device="cuda").manual_seed(47)
    v = (1 + torch.rand(M, device="cuda", generator=g)) * 2.0 ** torch.randint(-9, 9, (M,), device="cuda", generator=g)
    hi, mid, lo = pieces(v)
    assert torch.equal(hi + mid + lo, v) and torch.equal(lo.bfloat16().float(), lo) and (lo != 0).any()
    alpha, bias = torch.ones(3, device="cuda"), torch.zeros(N, device="cuda")
    bias[:n] = 300.0  # h^pre = 1, and no gradient through it
    one = torch.ones(N, n * C, device="cuda").to(dtype)
    wide = lambda t, *shape: t.reshape(-1, *(1 for _ in shape)).expand(-1, *shape).to(dtype).contiguous()

    def back(X, rows, dU, E):
        B = len(X)
        q, rms = torch.zeros(B, N, device="cuda"), torch.ones(B, device="cuda")
        return b4.pre_bwd(X, one, alpha, bias, q, rms, dU, None, rows.view(B, n, n).contiguous(), E)

    # token t's dH has entry t alone
    X = torch.randn(M, n, C, device="cuda", generator=g).to(dtype)
    dX = back(X, torch.diag(v), wide(-mid, C), wide(-hi, n, C))[0]
    assert torch.equal(dX.float(), lo[:, None, None].expand_as(dX))
    # three tokens an entry: the value, and its upper pieces taken away
    rows = torch.zeros(3 * M, M, device="cuda")
    for k, t in enumerate((v, -hi, -mid)):
        rows[torch.arange(M) * 3 + k, torch.arange(M)] = t
    dW = back(torch.ones(3 * M, n, C, device="cuda").to(dtype), rows, None, None)[1]
    assert torch.equal(dW[2 * n:].float(), lo[:, None].expand(-1, n * C)) and (dW[:2 * n] == 0).all()


def test_most_lanes():
    """Tokens times lanes a token past 2^32, which one dimension of a grid does not take."""
    n, B, C, part = 4, 1 << 25, 520, 1 << 19  # 65 chunks a row: two waves a token
    torch.cuda.empty_cache()
    free = torch.cuda.mem_get_info()[0]
    if free < 205 << 30:
        pytest.skip(f"needs 190 GiB of GPU memory, {free >> 30} are free")
    some, W, alpha, bias, _ = inputs(n, part, C, BF16, 49)
    X = torch.empty(B, n, C, dtype=BF16, device="cuda")
    X.view(B // part, *some.shape)[:] = some
    got = dict(zip(("U", "h", "H", "q", "rms"), b4.pre_fwd(X, W, alpha, bias)))
    torch.cuda.synchronize()
    for cut in (slice(0, 40), slice(B // 2 - 20, B // 2 + 20), slice(B - 40, B)):
        out, err, _ = pre_ref(X[cut], W, alpha, bias, 1e-6)
        for k in out:
            within(got[k][cut], out[k], err[k], f"{k} of tokens {cut.start}..")
    del X
    # every part's tokens are the first one's, up to the order of their sums: a bf16 step, an ulp's few of q
    for k, (tol, least) in dict(U=(2.0 ** -6, 1e-4), rms=(1e-6, 0.0), h=(1e-5, 1e-5)).items():
        parts = got[k].view(B // part, part, -1)
        ref = parts[0].float()
        for p in parts[1:]:
            assert ((p.float() - ref).abs() <= tol * ref.abs() + least).all(), k
    del got, parts, p, ref
    torch.cuda.empty_cache()  # the other tests', and other programs'


# rows of more than 512 chunks: several blocks a token in the forward's sum, several turns of a wave in the
# backward's dots; the widest ones leave the backward's products one share of the tokens (n C > 2048 waves'
# pieces), or are as wide as a row may be
WIDE = [(1, 4104), (33, 4104), (1, 8200), (33, 8200), (2049, 4104), (33, 16640), (33, 33288)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [4, 8])
@pytest.mark.parametrize("B,C", WIDE)
def test_wide_rows(n, B, C, dtype):
    C = C if dtype == BF16 else C // 2
    check(*inputs(n, B, C, dtype, 51), 1e-6, f"n={n} B={B} C={C} {dtype}")


@pytest.mark.parametrize("n,B,dtype", [(4, 3, BF16), (4, 65, F32), (8, 2, BF16)])
def test_widest_rows(n, B, dtype):
    """C = 2^20, the largest; 64 fp32 tokens' offsets are then next to what 32 bits hold."""
    check(*inputs(n, B, 1 << 20, dtype, 53), 1e-6, f"n={n} B={B} C=2^20 {dtype}")
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [4, 8])
def test_padding_tokens(n):
    """The tokens that fill the last stage of 32 count nothing in dW, whatever the last token holds:
    with q and rms given and G finite, an infinite value of the last token makes its column of dW
    infinite with the sign of G; read again for the padding, times its G of zero, it would make it
    NaN. (Nothing of dU's row goes through the value: dU is not given.)"""
    N, C, B = n * n + 2 * n, 40, 33
    X, W, alpha, bias, grads = inputs(n, B, C, F32, 55)
    q, rms = b4.pre_fwd(X, W, alpha, bias)[3:]
    clean = b4.pre_bwd(X, W, alpha, bias, q, rms, None, *grads[1:])[1]
    bad = X.clone()
    bad[B - 1, n - 1, 5] = float("inf")
    dX, dW, _, _ = b4.pre_bwd(bad, W, alpha, bias, q, rms, None, *grads[1:])
    col = torch.arange(n * C, device="cuda") == (n - 1) * C + 5
    assert torch.equal(dW[:, ~col], clean[:, ~col])
    # dH's rows: G = r alpha dH is not zero
    sign = torch.sign(alpha[2] * grads[2][B - 1].flatten())
    assert torch.equal(dW[2 * n:, col].flatten(), sign * float("inf"))
    assert torch.isfinite(dX[:B - 1]).all()


def test_gradient_of_one_token_stays_there():
    """A NaN in one token's gradient of the streams goes into that token's dX, and nowhere else."""
    X, W, alpha, bias, grads = inputs(4, 33, 64, BF16, 57)
    q, rms = b4.pre_fwd(X, W, alpha, bias)[3:]
    clean = b4.pre_bwd(X, W, alpha, bias, q, rms, *grads)
    E = grads[3].clone()
    E[32] = float("nan")
    dX, *others = b4.pre_bwd(X, W, alpha, bias, q, rms, *grads[:3], E)
    assert dX[32].isnan().all() and torch.equal(dX[:32], clean[0][:32])
    for a, b in zip(others, clean[1:]):
        assert torch.equal(a, b)
