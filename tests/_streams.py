"""float64 references of the streams' read (pre) and write (post), with the sizes of what their
outputs are sums of, from which the tests derive how far fp32 sums and roundings may be off.

u = 2^-24 is fp32's largest relative rounding error. A sum of m terms formed in any order is off by
at most (m - 1) u times the sum of the terms' magnitudes; the kernels' sums are trees of chains, of
which `depth` is the longest, which takes m's place. An approximate operation of the hardware (exp2,
reciprocal, reciprocal square root) is within 2 u.
"""
import torch

U32 = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def depth(terms: int) -> float:
    """Additions on the longest chain of a sum of `terms` products: the lanes' or tiles' own chain
    (a lane or a tile's column has every 32nd term or fewer of them, the matrix units add the
    products of one instruction in a chain of at most 32, and may drop what they round: twice u),
    then at most 64 partial sums of lanes, waves and shares."""
    return 2.0 * (terms / 32 + 32 + 64)


def pre_ref(X, W, alpha, bias, eps):
    """Outputs of pre in float64 and bounds of their errors before any rounding to a stream type:
    dict(U, h, H, q, rms), dict of the same names with bounds, and what the backward reuses."""
    n, C = X.shape[-2:]
    K, N = n * C, n * n + 2 * n
    x = X.double().reshape(-1, K)
    W, alpha, bias = W.double(), alpha.double(), bias.double()
    a = torch.cat([alpha[:1].expand(n), alpha[1:2].expand(n), alpha[2:].expand(n * n)])
    r = (x.square().mean(1, keepdim=True) + eps).rsqrt()
    q = r * (x @ W.t().contiguous())
    l = a * q + bias
    gate = torch.sigmoid(l[:, :2 * n])
    hp, h = gate[:, :n], 2 * gate[:, n:]
    Xd = x.view(-1, n, C)
    U = (hp[:, :, None] * Xd).sum(1)
    d = depth(K)
    e_r = (d / 2 + 4) * U32 * r  # half of |v|^2's relative error
    e_q = r * (x.abs() @ W.abs().t().contiguous()) * (d * U32) + q.abs() * (d / 2 + 6) * U32
    e_l = a.abs() * e_q + 2 * U32 * ((a * q).abs() + bias.abs())
    lg = l[:, :2 * n]
    # sigmoid' <= gate (1 - gate) near l; the exponent's rounding moves l by 2 u |l|
    e_gate = gate * (1 - gate) * (e_l[:, :2 * n] + 3 * U32 * lg.abs()) * 1.1 + 8 * U32 * gate
    e_U = (e_gate[:, :n, None] * Xd.abs()).sum(1) + (n + 1) * U32 * (hp[:, :, None] * Xd.abs()).sum(1)
    out = dict(U=U, h=h, H=l[:, 2 * n:].reshape(-1, n, n), q=q, rms=r[:, 0])
    err = dict(U=e_U, h=2 * e_gate[:, n:], H=e_l[:, 2 * n:].reshape(-1, n, n), q=e_q, rms=e_r[:, 0])
    return out, err, dict(x=x, W=W, a=a, r=r, q=q, gate=gate, e_r=e_r, e_q=e_q, e_gate=e_gate)


def pre_back_ref(ref, n, dU, dh, dH, E):
    """Gradients in float64 and bounds: (dX, dW, dalpha, dbias) twice; None inputs are zeros."""
    x, W, a, r, q, gate = (ref[k] for k in ("x", "W", "a", "r", "q", "gate"))
    B, K = x.shape
    N, C = W.shape[0], K // n
    zero = lambda t, *shape: torch.zeros(*shape, dtype=torch.float64, device=x.device) if t is None else t.double()
    dU, dh, dH, E = zero(dU, B, C), zero(dh, B, n), zero(dH, B, n, n), zero(E, B, n, C)
    dU, dh, dH, E = dU.reshape(B, C), dh.reshape(B, n), dH.reshape(B, n * n), E.reshape(B, K)
    X = x.view(B, n, C)
    dot, dot_abs = (X * dU[:, None]).sum(2), (X * dU[:, None]).abs().sum(2)
    s1 = gate * (1 - gate)
    up = torch.cat([dot, 2 * dh], 1)
    dl = torch.cat([up * s1, dH], 1)
    # errors of dl: the dot's, and that of gate (1 - gate), whose slope in gate is 1 - 2 gate
    e_up = torch.cat([depth(C) * U32 * dot_abs, torch.zeros_like(dh)], 1)
    e_s1 = (1 - 2 * gate).abs() * ref["e_gate"] + ref["e_gate"] ** 2 + 4 * U32 * s1
    e_dl = torch.cat([e_up * s1 + up.abs() * e_s1 + 2 * U32 * dl[:, :2 * n].abs(), torch.zeros_like(dH)], 1)
    G = r * a * dl
    e_G = r * a.abs() * e_dl + G.abs() * (ref["e_r"] / r + 4 * U32)
    s = (r / K) * (G * q).sum(1, keepdim=True)
    s_abs = (r / K) * (G * q).abs().sum(1, keepdim=True)
    e_s = (r / K) * (e_G * q.abs() + G.abs() * ref["e_q"]).sum(1, keepdim=True) + s_abs * (N + 8) * U32 \
        + s.abs() * ref["e_r"] / r
    hp = gate[:, :n].repeat_interleave(C, 1)
    e_hp = ref["e_gate"][:, :n].repeat_interleave(C, 1)
    dUk = dU.repeat(1, n)
    Wa = W.abs()
    dX = E + hp * dUk + G @ W - s * x
    mag = E.abs() + hp * dUk.abs() + G.abs() @ Wa + s_abs * x.abs()
    # G as two bf16 values: 2^-16 of it; sums over the rows
    e_dX = e_hp * dUk.abs() + e_G @ Wa + (G.abs() @ Wa) * (2.0 ** -16 + depth(N) * U32) + e_s * x.abs() + 8 * U32 * mag
    xa = x.abs()
    Gt = G.t().contiguous()
    dW = Gt @ x
    # a token's share of dW is off by its G, and sums over the tokens
    e_dW = e_G.t().contiguous() @ xa + (Gt.abs() @ xa) * (2.0 ** -16 + depth(B) * U32)
    dq = dl * q
    e_dq = e_dl * q.abs() + dl.abs() * ref["e_q"] + U32 * dq.abs()
    group = [slice(0, n), slice(n, 2 * n), slice(2 * n, N)]
    dalpha = torch.stack([dq[:, g].sum() for g in group])
    # lanes add a token's rows, then waves, turns and blocks add tokens
    d = depth(B) + 64
    e_dalpha = torch.stack([(e_dq[:, g] + d * U32 * dq[:, g].abs()).sum() for g in group])
    dbias, e_dbias = dl.sum(0), (e_dl + d * U32 * dl.abs()).sum(0)
    return (dX.view(B, n, C), dW, dalpha, dbias), (e_dX.view(B, n, C), e_dW, e_dalpha, e_dbias)


def within(got, ref, err, label, tiny=1e-30):
    """Every value of `got` within `err` of `ref`, plus one rounding to got's type (of a value that
    may itself be off by err)."""
    g, ref, err = got.double().reshape(ref.shape), ref, err
    slack = err + tiny
    if got.dtype == torch.bfloat16:
        slack = slack + ROUND[got.dtype] * (ref.abs() + slack)
    bad = ~((g - ref).abs() <= slack)
    worst = ((g - ref).abs() / slack).max().item() if g.numel() else 0.0
    print(f"  {label}: worst error / bound {worst:.3f}", flush=True)
    assert not bad.any(), f"{label}: {int(bad.sum())} of {bad.numel()} outside, worst {worst}"


def philox(counter, key):
    """One block of Philox 4x32-10 (Salmon et al. 2011) in Python's integers: counter of four
    words, key of two."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [b >> 32 ^ c[1] ^ k[0], b & 0xFFFFFFFF, a >> 32 ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(shape, p, seed, offset):
    """Which elements of Z stay: a bool tensor on the CPU."""
    numel = 1
    for s in shape:
        numel *= s
    words = []
    lo = lambda v: v & 0xFFFFFFFF
    for g in range((numel + 3) // 4):
        words += philox((lo(g), g >> 32, lo(offset), lo(offset >> 32)), (lo(seed), lo(seed >> 32)))
    return (torch.tensor(words[:numel], dtype=torch.int64) >= int(p * 2 ** 32)).reshape(shape)


def post_ref(P, X, h, Z, keep, p, dY=None):
    """Y in float64 from the projected P (its own errors are the projection's), or with dY the
    gradients (dX, dP, dh, dZ), each with its bound."""
    n, C = X.shape[-2:]
    P, X, h, Z = (t.double() for t in (P, X, h, Z))
    mult = keep.to(X.device).double() / (1.0 - p)
    # masked values do not count, whatever they are
    D = torch.where(mult > 0, Z * mult, torch.zeros_like(Z))
    if dY is None:
        Y = P @ X + h[:, :, None] * D[:, None]
        mag = P.abs() @ X.abs() + (h[:, :, None] * D[:, None]).abs()
        return Y, (2 * n + 4) * U32 * mag  # n + 1 terms; scale and its product with h rounded
    dY = dY.double()
    Pt = P.transpose(1, 2).contiguous()
    dX, e_dX = Pt @ dY, 2 * n * U32 * (Pt.abs() @ dY.abs())
    Xt = X.transpose(1, 2).contiguous()
    dP = dY @ Xt
    dh, dh_abs = (dY * D[:, None]).sum(2), (dY * D[:, None]).abs().sum(2)
    dZ = (h[:, :, None] * dY).sum(1) * mult
    e_dZ = (h[:, :, None] * dY).abs().sum(1) * mult * (2 * n + 4) * U32
    return (dX, dP, dh, dZ), (e_dX, None, (depth(C) + 4) * U32 * dh_abs, e_dZ)
