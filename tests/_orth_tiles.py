"""Sizes that run every form of the orthogonalisation's product kernel, and bounds that hold tile by tile."""
import torch

from tests._orth import COEFS, iterate, pieces, triples, turn, wide

F32, BF16 = torch.float32, torch.bfloat16

# [matrices, smaller side, larger side], the results' type, steps. What the first four kinds of products of each are made by:
# tiles of 64, 128 or 192 (192 not where the end reads more), in one group of waves, two or four. None is a whole
# number of tiles, so that tiles hang over at both edges.
ORTH = [((1, 92, 93), BF16, 5), ((20, 395, 446), BF16, 5), ((14, 723, 723), BF16, 5), ((1, 2007, 2111), BF16, 5),
        ((1, 3982, 4017), BF16, 5), ((45, 145, 248), BF16, 5), ((59, 147, 385), BF16, 5), ((1, 1326, 1707), BF16, 5),
        ((47, 144, 943), BF16, 5), ((1, 87, 90), F32, 5), ((13, 332, 439), F32, 5), ((31, 456, 497), F32, 5),
        ((1, 1997, 2051), F32, 5), ((36, 561, 789), F32, 5), ((55, 90, 129), F32, 5), ((60, 95, 532), F32, 5),
        ((1, 580, 3330), F32, 5), ((32, 301, 652), F32, 5), ((1, 87, 90), BF16, 8), ((1, 396, 2419), BF16, 8),
        ((1, 1545, 2444), BF16, 8), ((1, 650, 3026), BF16, 8)]
# updates whose steps run without X
STEP = [((1, 239, 1904), F32, 5), ((52, 140, 524), F32, 5), ((3, 1568, 2736), F32, 5), ((1, 2334, 3426), F32, 5)]


def sums(values, edge=32):
    """Sums over tiles of edge x edge values, of which the last ones take what is left too."""
    for axis in (1, 2):
        n = values.shape[axis]
        at = (torch.arange(n, device=values.device) // edge).clamp(max=max(n // edge, 1) - 1)
        shape = list(values.shape)
        shape[axis] = int(at.max()) + 1
        values = torch.zeros(shape, dtype=values.dtype, device=values.device).index_add_(axis, at, values)
    return values


def growth(c):
    """The most of |a + b t + c t^2| for t from 0 to 2, and at least one."""
    a, b, c = c
    at = [0.0, 2.0] + ([-0.5 * b / c] if c and 0 <= -0.5 * b / c <= 2 else [])
    return max(1.0, *(abs(a + b * t + c * t * t) for t in at))


def pairs_of(steps, coefs, dtype):
    """How many of the steps, from the first one on, take products of two fp16 pieces: all for fp32 results; for bf16 ones
    those in front of the last that multiply to 512 at most (and of the last one)."""
    if dtype == F32:
        return steps
    coefs = triples(coefs, steps)
    begin, product = steps - 1, growth(coefs[-1])
    while begin > 0 and product * growth(coefs[begin - 1]) <= 512:
        begin -= 1
        product *= growth(coefs[begin])
    return begin


def rounded(X, steps, coefs, pairs):
    """The steps with the stated roundings, as in tests/_orth.py: products of two fp16 pieces in the first `pairs` of them and
    of one in the others, the diagonals apart."""
    def apart(M):
        D = M.diagonal(dim1=1, dim2=2)
        return D, sum(pieces(M - torch.diag_embed(D)))

    Y = sum(pieces(X.float()))
    for k, (a, b, c) in enumerate(triples(coefs, steps)):
        def product(M, N):
            (mh, ml), (nh, nl) = pieces(M), pieces(N)
            return mh @ nh + (mh @ nl + ml @ nh) if k < pairs else mh @ nh

        D, R = apart(product(Y, turn(Y)))
        S = product(R, R) + (D[:, :, None] + D[:, None, :]) * R + torch.diag_embed(D * D)
        F, E = apart(b * (R + torch.diag_embed(D)) + c * S)
        Y = sum(pieces((a + F)[:, :, None] * Y + product(E, Y)))
    return Y.double()


def rounded_ref(G, steps, coefs, eps=0.0):
    """As orth_ref: float64's result, and per matrix three times the distance that these roundings take it, and one rounding
    of a step's terms in two pieces."""
    X, tall = wide(G, eps)
    ref = iterate(X, triples(coefs, steps))
    size = torch.linalg.vector_norm(ref, dim=(1, 2))
    bound = 3 * torch.linalg.vector_norm(rounded(X, steps, coefs, pairs_of(steps, coefs, G.dtype)) - ref, dim=(1, 2))
    return turn(ref) if tall else ref, bound + max(sum(abs(v) for v in c) for c in triples(coefs, steps)) * 2.0 ** -22 * size


def close_tiles(got, G, steps, label, times=1.0):
    """Each tile's error from float64's steps of a wide G, within what another draw of the roundings makes of it. They are of
    one size all over a matrix of independent values: three times those of `rounded` in this tile and on average (`times`
    that), one rounding of a step's terms as in orth_ref, and half a step of got's type in every value."""
    X, _ = wide(G, 1e-7)
    pairs = pairs_of(steps, COEFS, G.dtype)
    ref, model = iterate(X, [COEFS] * steps), rounded(X, steps, COEFS, pairs)
    half = {F32: 2.0 ** -24, BF16: 2.0 ** -8}[got.dtype]
    err, size = sums((got.double() - ref) ** 2).sqrt(), sums(ref ** 2).sqrt()
    own, count = sums((model - ref) ** 2), sums(torch.ones_like(ref))
    average = (model - ref).square().mean((1, 2), keepdim=True) * count
    terms = sum(abs(c) for c in COEFS) * (2.0 ** -22 if pairs == steps else 2.0 ** -11)
    bound = times * (3 * (own + average).sqrt() + terms * size)
    bound = bound + half * (size + bound)
    worst = (err / bound).max().item()
    print(f"  {label}: worst tile {worst:.2f} of its bound, which is up to {(bound / size).max().item():.1e} of its size", flush=True)
    assert (err <= bound).all(), f"{label}: {(err > bound).sum().item()} of {err.numel()} tiles, worst {worst:.2f} of its bound"
