"""float64 reference of the orthogonalisation, and how far the stated roundings take it from that.

The kernels' products are of values rounded to fp16 pieces (in units of 2^-12): for fp32 results of two
pieces each (hi hi + hi lo + lo hi), for bf16 results of one, with fp32 sums; X, A and E = b A + c A^2 are
kept as two pieces, the diagonals of A and E as fp32 numbers outside the products. `model` makes these roundings in torch's operations, in another order of sums. Its
distance from float64 is what the roundings cost for that matrix; they are random, so the kernels' own may
be another draw: three times it is allowed (of a Frobenius norm over few values, too). A matrix of very few
values can be lucky in the model; so one rounding of the terms of a step near s = 1, |a| + |b| + |c| = 10
times the factors' rounding (2^-22, 2^-11), is added, of the size of the result."""
import torch

COEFS = (3.4445, -4.7750, 2.0315)


def triples(coefs, steps):
    return [tuple(coefs)] * steps if not isinstance(coefs[0], (tuple, list)) else [tuple(c) for c in coefs]


def turn(M):
    return M.transpose(1, 2).contiguous()


def wide(G, eps):
    """As [matrices, smaller side, larger side] over their norms in float64, and whether turned."""
    G = G.double().reshape(-1, *G.shape[-2:])
    tall = G.shape[1] > G.shape[2]
    X = turn(G) if tall else G
    return X / (torch.linalg.vector_norm(X, dim=(1, 2), keepdim=True) + eps), tall


def iterate(X, coefs):
    for a, b, c in coefs:
        A = X @ turn(X)
        X = a * X + (b * A + c * (A @ A)) @ X
    return X


def pieces(M):
    s = M.float() * 4096
    hi = s.half().float()
    return hi / 4096, (s - hi).half().float() / 4096


def orth_ref(G, steps=5, coefs=COEFS, eps=1e-7, split=True):
    """The result in float64, and per matrix the bound of the error's Frobenius norm before the result is
    rounded to its type. split: the products of fp32 results."""
    coefs = triples(coefs, steps)
    X, tall = wide(G, eps)
    ref = iterate(X, coefs)

    def product(M, N):
        (mh, ml), (nh, nl) = pieces(M), pieces(N)
        return mh @ nh + (mh @ nl + ml @ nh) if split else mh @ nh

    def apart(M):
        D = M.diagonal(dim1=1, dim2=2)
        return D, M - torch.diag_embed(D)

    Y = sum(pieces(X.float()))
    for a, b, c in coefs:
        D, R = apart(product(Y, turn(Y)))
        R = sum(pieces(R))
        S = product(R, R) + (D[:, :, None] + D[:, None, :]) * R + torch.diag_embed(D * D)
        F, R = apart(b * (R + torch.diag_embed(D)) + c * S)
        Y = sum(pieces((a + F)[:, :, None] * Y + product(sum(pieces(R)), Y)))
    model = Y
    size = torch.linalg.vector_norm(ref, dim=(1, 2))
    terms = max(sum(abs(v) for v in c) for c in coefs)
    bound = 3 * torch.linalg.vector_norm(model.double() - ref, dim=(1, 2)) + terms * (2.0 ** -22 if split else 2.0 ** -11) * size
    return turn(ref) if tall else ref, bound


def close(got, ref, bound, label):
    """Per matrix, the error's Frobenius norm within the bound and half a step of got's type in every value."""
    half = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}[got.dtype]
    err = torch.linalg.vector_norm(got.double().reshape(ref.shape) - ref, dim=(1, 2))
    size = torch.linalg.vector_norm(ref, dim=(1, 2))
    most = bound + half * (size + bound)
    rel = lambda t: (t / size.clamp_min(1e-300)).max().item() if t.numel() else 0.0
    print(f"  {label}: error {rel(err):.2e} of the size, bound {rel(most):.2e}", flush=True)
    assert (err <= most).all(), f"{label}: error {rel(err):.2e}, bound {rel(most):.2e}"
