"""GPU parity of the layer norm (birkhoff4_norm_fwd / _norm_bwd) with float64, within the bounds of
tests/_norm.py, and of connect with a norm in front of its branch."""
import pytest
import torch

import paper_2606_07574_amd as b4
from tests._norm import norm_back_ref, norm_ref
from tests._streams import within

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5
EPS32 = torch.tensor(EPS, dtype=F32).item()  # what the kernels are given


def inputs(B, C, dtype, params, seed, offset=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)
    x = (normal(B, C) * (0.1 + 3 * torch.rand(B, 1, device="cuda", generator=g)) + offset * normal(C)).to(dtype)
    return x, (1 + 0.3 * normal(C)).to(params), (0.3 * normal(C)).to(params), normal(B, C).to(dtype)


def check(x, w, b, dy, label, eps=EPS32):
    print(label, flush=True)
    y, mean, rstd = b4.norm_fwd(x, w, b, eps)
    dx, dw, db = b4.norm_bwd(x, w, mean, rstd, dy)
    torch.cuda.synchronize()
    ref, err, saved = norm_ref(x, w, b, eps)
    for name, got, r, e in zip(("y", "mean", "rstd"), (y, mean, rstd), ref, err):
        within(got, r, e, name)
    ref, err = norm_back_ref(saved, dy)
    for name, got, r, e in zip(("dx", "dweight", "dbias"), (dx, dw, db), ref, err):
        within(got, r, e, name)


# one value, fewer than a chunk, every number of threads per row at both ends, rows in whole chunks and
# not, one row to more rows than the blocks take at once, rows that a block does not hold
SIZES = [(1, 1), (3, 1), (2, 3), (5, 7), (4, 8), (1, 4096), (70, 16), (2600, 24), (33, 127), (300, 128), (65, 129), (40, 256),
         (301, 257), (17, 1000), (1100, 512), (9, 1023), (2050, 1024), (30, 2052), (600, 513), (600, 2049), (6, 4100), (300, 4097),
         (5, 8192), (270, 8191), (3, 8193), (2, 20001), (1, 65536), (3, 16384),
         (2, 16385)]


@pytest.mark.parametrize("types", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)], ids=["f32", "mixed", "bf16", "f32bf16"])
@pytest.mark.parametrize("B,C", SIZES)
def test_sizes(B, C, types):
    check(*inputs(B, C, *types, 7 * B + C), f"B={B} C={C} {types}")


def test_widest():
    check(*inputs(2, 1 << 20, BF16, BF16, 5), "2^20 wide")


@pytest.mark.parametrize("C", [1024, 1021, 9000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_offsets(C, dtype):
    """A common offset far above the spread: the bounds say what remains of it."""
    check(*inputs(50, C, dtype, F32, 3, offset=300.0), f"offset C={C}")
    x, w, b, dy = inputs(50, C, dtype, F32, 4)
    check((x.float() * 1e-6).to(dtype), w, b, dy, f"small C={C}")
    check((x.float() * 1e8).to(dtype), w, b, dy, f"large C={C}")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_without_parameters(dtype):
    x, w, b, dy = inputs(37, 200, dtype, F32, 6)
    for p in ((None, None), (w, None), (None, b)):
        y, mean, rstd = b4.norm_fwd(x, *p, EPS32)
        dx, dw, db = b4.norm_bwd(x, p[0], mean, rstd, dy)
        ref, err, saved = norm_ref(x, *p, EPS32)
        within(y, ref[0], err[0], "y")
        ref, err = norm_back_ref(saved, dy)
        for name, got, r, e in zip(("dx", "dweight", "dbias"), (dx, dw, db), ref, err):
            within(got, r, e, name)


def test_constant_rows():
    """No spread: y is the bias, and eps alone holds the derivative."""
    x = torch.full((5, 96), 3.0, device="cuda")
    _, w, b, dy = inputs(5, 96, F32, F32, 8)
    y, mean, rstd = b4.norm_fwd(x, w, b, EPS32)
    assert torch.equal(y, b.expand(5, 96)) and (mean == 3).all()
    check(x, w, b, dy, "constant rows")


@pytest.mark.parametrize("C", [40, 1000, 1023, 4096, 9001])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_bad_rows_alone(C, bad):
    """A row with a NaN or infinity gives NaN there and in the sums, and nothing elsewhere."""
    x, w, b, dy = inputs(70, C, BF16, F32, 9)
    y0, m0, s0 = b4.norm_fwd(x, w, b)
    d0 = b4.norm_bwd(x, w, m0, s0, dy)
    rows = [0, 33, 69]
    x[rows, [0, C // 2, C - 1]] = bad
    y, m, s = b4.norm_fwd(x, w, b)
    dx, dw, db = b4.norm_bwd(x, w, m, s, dy)
    good = torch.ones(70, dtype=torch.bool, device="cuda")
    good[rows] = False
    assert torch.equal(y[good], y0[good]) and torch.equal(dx[good], d0[0][good]) and torch.equal(db, d0[2])
    assert y[rows].isnan().all() and dx[rows].isnan().all() and dw.isnan().all()


@pytest.mark.parametrize("C", [16, 1023, 9000])
def test_no_rows(C):
    x, w, b, dy = inputs(0, C, BF16, BF16, 9)
    y, mean, rstd = b4.norm_fwd(x, w, b)
    assert y.shape == (0, C) and mean.shape == (0,)
    dx, dw, db = b4.norm_bwd(x, w, mean, rstd, dy)
    assert dx.shape == (0, C) and (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,C", [(7, 45), (3, 1023), (5, 9001), (300, 130)])
def test_nothing_behind(B, C, dtype):
    """What lies right in front of and behind every output stays as it was."""
    x, w, b, dy = inputs(B, C, dtype, F32, 11)
    lib, stream = b4.lib(), torch.cuda.current_stream().cuda_stream
    mark, pad = -7.0, 64

    def guarded(numel, dt):
        whole = torch.full((numel + 2 * pad,), mark, dtype=dt, device="cuda")
        return whole, whole[pad:pad + numel]

    ys, ms, rs, dxs, dws, dbs = (guarded(*k) for k in ((B * C, dtype), (B, F32), (B, F32), (B * C, dtype), (C, F32), (C, F32)))
    code = b4.BF16 if dtype == BF16 else b4.F32
    work = torch.empty(lib.birkhoff4_norm_work(B, C, code), dtype=torch.uint8, device="cuda")
    assert lib.birkhoff4_norm_fwd(x.data_ptr(), code, w.data_ptr(), b.data_ptr(), b4.F32, EPS, ys[1].data_ptr(),
                                  ms[1].data_ptr(), rs[1].data_ptr(), B, C, stream) == 0
    assert lib.birkhoff4_norm_bwd(x.data_ptr(), code, w.data_ptr(), b4.F32, ms[1].data_ptr(), rs[1].data_ptr(), dy.data_ptr(),
                                  dxs[1].data_ptr(), dws[1].data_ptr(), dbs[1].data_ptr(), work.data_ptr(), work.numel(), B, C,
                                  stream) == 0
    torch.cuda.synchronize()
    y, m, s = b4.norm_fwd(x, w, b, EPS)
    for (whole, part), ref in zip((ys, ms, rs, dxs, dws, dbs), (y, m, s, *b4.norm_bwd(x, w, m, s, dy))):
        assert torch.equal(part, ref.reshape(-1))
        assert (whole[:pad] == mark).all() and (whole[pad + part.numel():] == mark).all()


def test_far_rows():
    """Rows beyond 2^31 values and 2^32 bytes."""
    B, C = (1 << 31) // 4096 + 700, 4096
    x = torch.empty(B, C, dtype=BF16, device="cuda")
    tail, w, b, dyt = inputs(400, C, BF16, F32, 12)
    x.fill_(1.0)
    x[-400:] = tail
    y, mean, rstd = b4.norm_fwd(x, w, b, EPS32)
    ref, err, saved = norm_ref(tail, w, b, EPS32)
    within(y[-400:], ref[0], err[0], "y")
    del y
    dy = torch.zeros_like(x)
    dy[-400:] = dyt
    dx, dw, db = b4.norm_bwd(x, w, mean, rstd, dy)
    ref, err = norm_back_ref(saved, dyt)
    within(dx[-400:], ref[0], err[0], "dx")
    assert (dx[:1000] == 0).all()
    # most rows add nothing: the bounds of the 400 hold
    within(dw, ref[1], err[1], "dweight")
    within(db, ref[2], err[2], "dbias")


@pytest.mark.parametrize("params", [F32, BF16])
def test_autograd(params):
    """Strided and misplaced inputs, leading axes, and gradients that only some inputs want."""
    g = torch.Generator(device="cuda").manual_seed(13)
    flat = torch.randn(2 * 5 * 33 * 2 + 1, device="cuda", generator=g)
    x = flat[1:].view(2, 5, 66)[..., ::2].detach().requires_grad_(True)
    buf = torch.randn(67, device="cuda", generator=g).to(params)
    w, b = buf[1:34].detach().requires_grad_(True), buf[34:].detach().requires_grad_(True)
    dy = torch.randn(2, 33, 5, device="cuda", generator=g).transpose(1, 2)
    y = b4.norm(x, w, b, EPS32)
    grads = torch.autograd.grad(y, (x, w, b), dy)
    ref, err, saved = norm_ref(x.detach(), w.detach(), b.detach(), EPS32)
    within(y.detach(), ref[0], err[0], "y")
    ref, err = norm_back_ref(saved, dy)
    for got, r, e in zip(grads, ref, err):
        within(got, r, e, "grad")
        assert got.dtype in (F32, params)
    for k, t in enumerate((x, w, b)):
        args = [a.detach() for a in (x, w, b)]
        args[k].requires_grad_(True)
        alone, = torch.autograd.grad(b4.norm(*args, EPS32), args[k], dy)
        assert torch.equal(alone, grads[k])
    with torch.no_grad():
        assert torch.equal(b4.norm(x, w, b, EPS32), y)
    with pytest.raises(RuntimeError):
        gx, = torch.autograd.grad(b4.norm(x, w, b), x, dy, create_graph=True)
        gx.sum().backward()


def test_refusals():
    x, w, b, dy = inputs(4, 32, BF16, F32, 14)
    for bad, error in (((x.half(), w, b), TypeError), ((x.t(), w[:4], b[:4]), ValueError), ((x, w[:31], b), ValueError),
                       ((x, w, b.bfloat16()), TypeError), ((x, w.double(), None), TypeError), ((x, w.cpu(), b), b4.Birkhoff4Error),
                       ((x[:, :0], None, None), ValueError), ((x, w, b, -1.0), b4.Birkhoff4Error)):
        with pytest.raises(error):
            b4.norm_fwd(*bad)
    y, m, s = b4.norm_fwd(x, w, b)
    for bad, error in (((x, w, m, s, dy[:3]), ValueError), ((x, w, m, s, dy.float()), TypeError),
                       ((x, w, m[:3], s, dy), ValueError), ((x, w, m, s.bfloat16(), dy), TypeError)):
        with pytest.raises(error):
            b4.norm_bwd(*bad)


@pytest.mark.parametrize("B,C", [(3, 500), (700, 1024), (5, 9000)])
def test_graphs(B, C):
    """Two captured passes with workspaces of their own, replayed between eager work, give the eager bits."""
    sets = [inputs(B, C, BF16, F32, 20 + k) for k in range(3)]
    static = [[t.clone() for t in sets[0]] for _ in range(2)]

    def both(x, w, b, dy):
        y, m, s = b4.norm_fwd(x, w, b)
        return (y, *b4.norm_bwd(x, w, m, s, dy))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(*static[0])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for k in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[k]):
            outs.append(both(*static[k]))
    for turn in range(3):
        for k in range(2):
            for d, src in zip(static[k], sets[(turn + k) % 3]):
                d.copy_(src)
        refs = [both(*sets[(turn + k) % 3]) for k in range(2)]
        torch.cuda.synchronize()
        for rep in range(2):
            for g in graphs:
                g.replay()
            torch.cuda.synchronize()
            for ref, out in zip(refs, outs):
                assert all(torch.equal(r, o) for r, o in zip(ref, out))
                for o in out:
                    o.fill_(float("nan"))


def test_other_stream():
    x, w, b, dy = inputs(900, 512, F32, F32, 15)
    ref = b4.norm_fwd(x, w, b)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = b4.norm_fwd(x, w, b)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(ref, got))


@pytest.mark.parametrize("n", [4, 8])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_connect(n, dtype):
    """connect with a norm is pre, norm, the branch and post, values and gradients."""
    g = torch.Generator(device="cuda").manual_seed(16)
    B, C, R = 40, 64, n * n + 2 * n
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)
    X, W = normal(B, n, C).to(dtype), (normal(R, n * C) / (n * C) ** 0.5).to(dtype)
    leaves = [X, W, 1 + 0.1 * normal(3), 0.1 * normal(R), 1 + 0.1 * normal(C), 0.1 * normal(C)]
    for t in leaves:
        t.requires_grad_(True)
    dY = normal(B, n, C).to(dtype)

    def parts(X, W, alpha, bias, w, b):
        U, h, H, X = b4.pre(X, W, alpha, bias)
        return b4.post(H, X, h, torch.tanh(b4.norm(U, w, b)))

    whole = lambda X, W, alpha, bias, w, b: b4.connect(X, W, alpha, bias, torch.tanh, norm=(w, b))
    Y, Z = whole(*leaves), parts(*leaves)
    assert torch.equal(Y, Z) and not torch.equal(Y, b4.connect(*leaves[:4], torch.tanh))
    for a, c in zip(torch.autograd.grad(Y, leaves, dY), torch.autograd.grad(Z, leaves, dY)):
        assert torch.equal(a, c)
    with torch.no_grad():
        assert torch.equal(whole(*leaves), Y)
        assert torch.equal(b4.connect(*leaves[:4], torch.tanh, norm=(None, None)),
                           b4.connect(*leaves[:4], lambda U: torch.tanh(b4.norm(U))))
