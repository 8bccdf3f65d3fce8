"""Matrices whose rows are not independent, exactly so in their type, and the orthogonalisation's float64 result for
them: with G = Q K for Q of orthonormal columns and K of full rank, every step is Q times that of K, so K's steps
alone are taken (those of G in float64 would lose all digits where steps grow a rounding of a zero singular value)."""
import torch

from tests._orth import COEFS, iterate, triples, turn, wide

CUBIC = (1.5, -0.5, 0.0)
PAIRS = [(4.0, -6.0, 2.5), (2.0, -1.5, 0.5)]  # singular values stay below 1.4


def dependent(m, n, dtype, kind, seed, matrices=1, device="cuda"):
    """(G [matrices, m, n] in dtype, Q, K): every row twice, or of rank one or three with small whole numbers."""
    g = torch.Generator().manual_seed(seed)
    if kind == "twice":
        X = torch.randn(matrices, (m + 1) // 2, n, generator=g).to(dtype).double()
        L = torch.eye((m + 1) // 2, dtype=torch.float64).repeat_interleave(2, 0)[:m].expand(matrices, -1, -1)
    else:
        r = {"one": 1, "three": 3}[kind]
        top = 8 if r == 1 else 5  # sums of products of them have no more than bf16's 8 bits
        L = torch.randint(-top + 1, top, (matrices, m, r), generator=g).double()
        X = torch.randint(-top + 1, top, (matrices, r, n), generator=g).double()
        L[:, torch.arange(r), torch.arange(r)] += 1.0 + top // 2  # none is zero
        X[:, torch.arange(r), torch.arange(r)] += 1.0 + top // 2
    G = torch.matmul(L, X)
    assert torch.equal(G.to(dtype).double(), G)
    Q, R = torch.linalg.qr(L)
    return G.to(dtype).to(device), Q.to(device), torch.matmul(R, X).to(device)


def dependent_ref(Q, K, steps, coefs=COEFS, eps=0.0):
    """With the coefficients as the kernels are given them, fp32 numbers."""
    coefs = [tuple(torch.tensor(c, dtype=torch.float32).tolist()) for c in triples(coefs, steps)]
    X = K / (torch.linalg.vector_norm(K, dim=(1, 2), keepdim=True) + eps)
    return torch.matmul(Q, iterate(X, coefs))


def fades(m, n, dtype, seed, last=1e-7, device="cuda"):
    """Singular values from one down to `last`, evenly in their logarithm."""
    g = torch.Generator().manual_seed(seed)
    U, _ = torch.linalg.qr(torch.randn(m, m, generator=g, dtype=torch.float64))
    V, _ = torch.linalg.qr(torch.randn(n, m, generator=g, dtype=torch.float64))
    s = torch.logspace(0, torch.log10(torch.tensor(last)).item(), m, dtype=torch.float64)
    return torch.matmul(U * s, turn(V[None])[0]).to(dtype)[None].to(device)


def carried(G, steps, coefs=COEFS, eps=0.0):
    """Per matrix, the Frobenius norm of what later steps make of one rounding of each step's terms, (|a| + |b| + |c|) 2^-22
    of every singular value: an error of a value s ahead of a step is p'(s) = a + 3 b s^2 + 5 c s^4 times as large behind
    it. The usual steps never come to rest (p' = -1.6 where p(s) = s), so that after 40 of them a value near an edge
    has been multiplied by 10^5 and more; a draw of the roundings says nothing of another draw there."""
    coefs = triples(coefs, steps)
    X, _ = wide(G, eps)
    s = torch.linalg.svdvals(X)
    path, error = [s], torch.zeros_like(s)
    for a, b, c in coefs:
        path.append(a * path[-1] + b * path[-1] ** 3 + c * path[-1] ** 5)
    for k, (a, b, c) in enumerate(coefs):
        at = path[k]
        error = error * (a + 3 * b * at ** 2 + 5 * c * at ** 4).abs() + (abs(a) + abs(b) + abs(c)) * 2.0 ** -22 * path[k + 1].abs()
    return torch.linalg.vector_norm(error.clamp(max=2.0), dim=1)
