"""Performance cases of what a hyper-connection layer is trained with around its read and write:
the layer norm of the branch's input, and the orthogonalised update of weight matrices, among them
the coefficients' matrices W [n^2 + 2 n, n C] of the read.

Every case names an operator, a direction and its sizes; ``prepare`` draws the inputs on the
GPU from a seed, ``run`` makes one pass through the operator (``own``: through the public entry
points of ``paper_2606_07574_amd``; otherwise in elementary torch operations), ``exact`` gives
the same results in float64.

Operators
  norm   y = (x - mean x) / sqrt(var x + eps) * weight + bias over the last axis of x [B, C], and
         the gradients of x, weight and bias.
  orth   the matrices G [L, m, n] taken towards their nearest (semi-)orthogonal ones by Newton-Schulz
         products: X = G / (|G|_F + eps), then five times X <- a X + (b A + c A^2) X with A = X X^T
         (for m > n from the other side, which is the same of the transpose).
  step   an update with momentum: M <- mu M + G, U = G + mu M, W <- (1 - lr decay) W - lr scale orth(U),
         scale = sqrt(max(1, m / n)).
"""
import math

import torch

own = False

F32, BF16 = "f32", "bf16"
DTYPES = {F32: torch.float32, BF16: torch.bfloat16}
NORM_EPS, ORTH_EPS = 1e-5, 1e-7
COEFS, STEPS = (3.4445, -4.7750, 2.0315), 5
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.1


def listed():
    return [
        # the branch's input for one new token: latency alone
        dict(name="norm_token", op="norm", train=False, dtype=BF16, params=BF16, B=1, C=4096),
        # a training micro-batch of 32 K tokens of width 4096, both directions, fp32 parameters
        dict(name="norm_train", op="norm", train=True, dtype=BF16, params=F32, B=32768, C=4096),
        # fp32, a ragged number of tokens
        dict(name="norm_f32", op="norm", train=True, dtype=F32, params=F32, B=4097, C=1000),
        # an odd width, whose rows begin at any element
        dict(name="norm_odd", op="norm", train=True, dtype=BF16, params=BF16, B=8191, C=1023),
        # the gradient of one layer's coefficients' matrix, four streams of 4096: latency
        dict(name="orth_read4", op="orth", dtype=F32, L=1, m=24, n=16384),
        # those of 32 layers with eight streams at once
        dict(name="orth_read8", op="orth", dtype=BF16, L=32, m=80, n=32768),
        # a square projection of a branch
        dict(name="orth_square", op="orth", dtype=BF16, L=1, m=4096, n=4096),
        # ragged sizes in fp32, rows that begin at any element
        dict(name="orth_ragged", op="orth", dtype=F32, L=1, m=1000, n=2565),
        # the heads' matrices of a branch, tall and many
        dict(name="orth_heads", op="orth", dtype=BF16, L=48, m=512, n=128),
        # the whole update of one coefficients' matrix
        dict(name="step_read4", op="step", dtype=F32, weights=F32, L=1, m=24, n=16384),
        # a wide branch's weights: bf16 gradients, fp32 weights
        dict(name="step_wide", op="step", dtype=BF16, weights=F32, L=1, m=10240, n=2560),
        # the same projection of six layers, bf16 weights
        dict(name="step_layers", op="step", dtype=BF16, weights=BF16, L=6, m=1024, n=1024),
    ]


def _log(rng, lo, hi):
    """A whole number spread evenly over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "orth", "orth", "step", "step"])
    dtype, other = rng.choice([F32, BF16]), rng.choice([F32, BF16])
    if op == "norm":
        C = _log(rng, 16, 8192)
        return dict(op=op, train=rng.random() < 0.7, dtype=dtype, params=F32 if dtype == F32 else other,
                    B=_log(rng, 1, min(32768, (1 << 27) // C)), C=C)
    case = dict(op=op, dtype=dtype)
    if op == "step":
        case["weights"] = other
    if rng.random() < 0.3:  # coefficients' matrices of a few layers
        streams = rng.choice([4, 8])
        m, n = streams * streams + 2 * streams, streams * 8 * _log(rng, 16, 512)
    else:
        m, n = _log(rng, 16, 4096), _log(rng, 16, 8192)
    # no more products than the largest listed case's, and no more values than a quarter of the largest's
    small = min(m, n)
    most = min(1.3e12 / (STEPS * small * small * (3 * max(m, n) + small)), (1 << 25) / (m * n))
    if most < 1.0:
        m = max(16, int(m * most))
        most = 1.0
    return dict(case, L=_log(rng, 1, min(48, most)), m=m, n=n)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]

    def normal(*shape, dtype=torch.float32):
        return torch.randn(*shape, device=dev, generator=g, dtype=dtype)

    s = {"case": case}
    if case["op"] == "norm":
        B, C, params = case["B"], case["C"], DTYPES[case["params"]]
        # tokens of different sizes around a common offset
        s["x"] = normal(B, C, dtype=dt) * torch.exp(0.5 * normal(B, 1)).to(dt) + normal(C, dtype=dt)
        s["weight"] = (1.0 + 0.1 * normal(C)).to(params)
        s["bias"] = (0.1 * normal(C)).to(params)
        if case["train"]:
            s["dy"] = normal(B, C, dtype=dt)
            for k in ("x", "weight", "bias"):
                s[k].requires_grad_(True)
        return s
    L, m, n = case["L"], case["m"], case["n"]

    def gradient(dtype, size):
        """A gradient: a few strong directions and much that is spread out."""
        r = min(m, n, 16)
        strong = torch.exp(-0.25 * torch.arange(r, device=dev, dtype=torch.float32))
        left, right = normal(L, m, r) * strong, normal(L, r, n)
        return (size * (torch.matmul(left, right) + 0.3 * normal(L, m, n))).to(dtype)

    s["G"] = gradient(dt, 1e-3)
    if case["op"] == "step":
        s["W"] = normal(L, m, n, dtype=DTYPES[case["weights"]]) / math.sqrt(n)
        s["M"] = gradient(torch.float32, 1e-2)
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2606_07574_amd as b4

    case = s["case"]
    if case["op"] == "norm":
        if not case["train"]:
            return b4.norm_fwd(s["x"], s["weight"], s["bias"], NORM_EPS)
        inputs = [s["x"], s["weight"], s["bias"]]
        y = b4.norm(*inputs, NORM_EPS)
        return (y.detach(),) + torch.autograd.grad(y, inputs, s["dy"])
    if case["op"] == "orth":
        return b4.orth(s["G"], STEPS, COEFS, ORTH_EPS)
    b4.orth_step(s["W"], s["G"], s["M"], LR, MOMENTUM, nesterov=True, decay=DECAY, steps=STEPS, coefs=COEFS, eps=ORTH_EPS)
    return s["W"], s["M"]


def _run_plain(s):
    with torch.no_grad():
        if s["case"]["op"] == "norm":
            return _norm_plain(s)
        if s["case"]["op"] == "orth":
            return _orth_plain(s["G"].float()).to(s["G"].dtype)
        W, G, M = s["W"], s["G"].float(), s["M"]
        M.mul_(MOMENTUM).add_(G)
        O = _orth_plain(G + MOMENTUM * M)
        W.copy_((1.0 - LR * DECAY) * W.float() - (LR * _scale(s["case"])) * O)
        return W, M


def _scale(case):
    return math.sqrt(max(1.0, case["m"] / case["n"]))


def _norm_plain(s):
    x, w = s["x"].float(), s["weight"].float()
    dt, params = s["x"].dtype, s["weight"].dtype
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + NORM_EPS)
    xhat = d * rstd
    y = (xhat * w + s["bias"].float()).to(dt)
    if not s["case"]["train"]:
        return y, mean[:, 0], rstd[:, 0]
    dy = s["dy"].float()
    g = dy * w
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return y, dx.to(dt), (dy * xhat).sum(0).to(params), dy.sum(0).to(params)


def _orth_plain(G):
    """The iteration in 32 bits, from the side on which A is smaller."""
    a, b, c = COEFS
    tall = G.shape[1] > G.shape[2]
    X = G.transpose(1, 2).contiguous() if tall else G
    X = X / (torch.sqrt((X * X).sum((1, 2), keepdim=True)) + ORTH_EPS)
    for _ in range(STEPS):
        A = torch.matmul(X, X.transpose(1, 2).contiguous())
        X = a * X + torch.matmul(b * A + c * torch.matmul(A, A), X)
    return X.transpose(1, 2).contiguous() if tall else X


def work(case):
    """Bytes: each input read and each output written once. Operations of the products: two for a
    multiplication and an addition, one for those of a symmetric result, of which half is needed;
    where it is less, one A, the iteration on factors of its size and one product with X."""
    size = 2 if case["dtype"] == BF16 else 4
    if case["op"] == "norm":
        B, C, params = case["B"], case["C"], 2 if case["params"] == BF16 else 4
        nbytes, flops = 2 * B * C * size + 2 * C * params, 7 * B * C
        if case["train"]:
            nbytes += 2 * B * C * size + 2 * C * params
            flops += 14 * B * C
        else:
            nbytes += 8 * B
        return {"bytes": nbytes, "flops": flops}
    L, values = case["L"], case["L"] * case["m"] * case["n"]
    small, large = min(case["m"], case["n"]), max(case["m"], case["n"])
    every = STEPS * small * small * (3 * large + small)
    once = 3 * small * small * large + STEPS * 4 * small ** 3
    flops = L * min(every, once) + 4 * values
    if case["op"] == "orth":
        return {"bytes": 2 * values * size, "flops": flops}
    # W and M are read and written
    return {"bytes": values * (size + 8 + 2 * (2 if case["weights"] == BF16 else 4)), "flops": flops + 6 * values}


# ---------------------------------------------------------------------------
# The same in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _norm_exact(s)
    G = s["G"].double()
    if case["op"] == "orth":
        return _orth_exact(G)
    M = s["M"].double() * MOMENTUM + G
    O = _orth_exact(G * (1 + MOMENTUM) + (MOMENTUM * MOMENTUM) * s["M"].double())
    return s["W"].double() * (1 - LR * DECAY) - O * (LR * _scale(case)), M


def _norm_exact(s):
    """From sums of powers and of products, rows in parts; the derivative as that of a projection
    off the vectors 1 and x, each of which is of length sqrt(C) after the normalisation."""
    case = s["case"]
    C, w, bias = case["C"], s["weight"].detach().double(), s["bias"].detach().double()
    rows, dw, db = [], 0.0, 0.0
    step = max(1, (1 << 24) // C)
    for a in range(0, case["B"], step):
        x = s["x"].detach()[a:a + step].double()
        s1, s2 = x.sum(1), torch.linalg.vector_norm(x, dim=1) ** 2
        mean = s1 / C
        sd = ((s2 - s1 * mean) / C + NORM_EPS).sqrt()
        xhat = torch.addcmul(-(mean / sd)[:, None], x, (1 / sd)[:, None])
        y = torch.addcmul(bias, xhat, w).float()  # far past the stream's rounding
        if not case["train"]:
            rows.append((y, mean, 1 / sd))
            continue
        dy = s["dy"][a:a + step].double()
        g = dy * w
        basis = torch.stack([torch.ones_like(xhat), xhat], 1)
        coef = torch.matmul(basis, g[:, :, None]) / C
        dx = (g - torch.matmul(coef.transpose(1, 2).contiguous(), basis)[:, 0]) / sd[:, None]
        rows.append((y, dx.float()))
        dw = dw + torch.einsum("bc,bc->c", dy, xhat)
        db = db + dy.sum(0)
    outs = tuple(torch.cat(k) for k in zip(*rows))
    return outs + ((dw, db) if case["train"] else ())


def _orth_exact(G):
    """X after k steps is a polynomial in A_0 = X_0 X_0^T times X_0: the iteration runs on the
    polynomials' values, A_k = p_k^2 A_(k-1) and F_k = p_k F_(k-1), which all commute."""
    a, b, c = COEFS
    tall = G.shape[1] > G.shape[2]
    X = G.transpose(1, 2).contiguous() if tall else G
    X = X / (torch.linalg.vector_norm(X, dim=(1, 2), keepdim=True) + ORTH_EPS)
    eye = torch.eye(X.shape[1], dtype=X.dtype, device=X.device)
    A, F = torch.matmul(X, X.transpose(1, 2).contiguous()), eye.expand(X.shape[0], -1, -1)
    for _ in range(STEPS):
        p = torch.matmul(A, c * A + b * eye) + a * eye
        F = torch.matmul(p, F)
        A = torch.matmul(p, torch.matmul(p, A))
    O = torch.matmul(F, X)
    return O.transpose(1, 2).contiguous() if tall else O
