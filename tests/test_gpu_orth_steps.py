"""GPU parity of the orthogonalisation over its whole range of steps, where rows depend on each other or singular
values fade away: what steps make of the roundings of a zero singular value is not bounded by the result's size
unless the kernels see to it."""
import pytest
import torch

import paper_2606_07574_amd as b4
from tests._orth import COEFS, close, orth_ref, turn
from tests._orth_rank import CUBIC, PAIRS, carried, dependent, dependent_ref, fades
from tests._orth_tiles import rounded_ref

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def narrow_bound(ref, m, steps):
    """With a side of at most 80 all is done in 64 bits, P = m rounded up to 16. The steps' polynomial F stays below
    64 / sqrt(2 P^1.5 2^-53) (what singular values are held above, and what the steps before grow them by), and a
    step rounds P products of its values with some up to four (the largest of the steps' coefficients a); a
    product with G rounds them once more."""
    P = (m + 15) // 16 * 16
    largest = 64 / (2 * P ** 1.5 * 2.0 ** -53) ** 0.5
    return torch.linalg.vector_norm(ref, dim=(1, 2)) * (steps + 1) * 4 * P * 2.0 ** -53 * largest


RUNS = [(6, COEFS), (8, COEFS), (10, COEFS), (14, COEFS), (18, COEFS), (25, COEFS), (64, COEFS), (25, CUBIC), (56, CUBIC),
        (10, [COEFS] * 8 + [(2.0, -1.5, 0.5)] * 2), (16, PAIRS * 6 + [CUBIC] * 4), (9, [(0.25, 0.5, 0.0)] * 4 + [(2.0, 0.5, -0.5)] * 5)]


def run_id(run):
    return f"{run[0]}x{'default' if run[1] is COEFS else 'cubic' if run[1] is CUBIC else 'mixed'}"


@pytest.mark.parametrize("run", RUNS, ids=run_id)
@pytest.mark.parametrize("kind", ["twice", "one", "three"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(24, 1024), (80, 2056), (7, 130), (33, 6000)])
def test_dependent_rows(m, n, dtype, kind, run):
    steps, coefs = run
    G, Q, K = dependent(m, n, dtype, kind, m + steps, matrices=2)
    ref = dependent_ref(Q, K, steps, coefs)
    bound = narrow_bound(ref, m, steps)
    label = f"{m} x {n} {dtype} {kind} {run_id(run)}"
    print(label, flush=True)
    close(b4.orth(G, steps, coefs, 0.0), ref, bound, label)
    close(b4.orth(turn(G), steps, coefs, 0.0), turn(ref), bound, label + " tall")


@pytest.mark.parametrize("w_dtype", [F32, BF16], ids=["wf32", "wbf16"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind", ["twice", "one"])
@pytest.mark.parametrize("steps", [10, 25, 64])
def test_update_of_dependent_rows(steps, kind, dtype, w_dtype):
    """The direction itself, read off weights of zero."""
    for tall in (False, True):
        G, Q, K = dependent(24, 1500, dtype, kind, steps, matrices=3)
        ref = dependent_ref(Q, K, steps)
        G, ref = (turn(G), turn(ref)) if tall else (G, ref)
        for momentum, nesterov in ((0.0, False), (0.5, True)):
            W, M = torch.zeros(G.shape, dtype=w_dtype, device="cuda"), torch.zeros(G.shape, device="cuda")
            b4.orth_step(W, G, M, -1.0, momentum, nesterov, scale=1.0, steps=steps, eps=0.0)
            assert torch.equal(M, G.float())
            close(W, ref, narrow_bound(ref, 24, steps), f"{steps} {kind} {dtype} {w_dtype} tall={tall}")


@pytest.mark.parametrize("run", [(8, COEFS), (10, COEFS), (12, COEFS), (25, COEFS), (64, COEFS), (25, CUBIC), (56, CUBIC)], ids=run_id)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(24, 1024), (80, 2056)])
def test_fading_rows(m, n, dtype, run):
    """Singular values down to 1e-7 (bf16: as far as its rounding lets them): no further off than products of two
    fp16 pieces take it, and of the size of an orthogonal matrix."""
    steps, coefs = run
    G = fades(m, n, dtype, m)
    ref, bound = orth_ref(G, steps, coefs, 0.0, split=dtype == F32)
    O = b4.orth(G, steps, coefs, 0.0)
    close(O, ref, bound, f"{m} x {n} {dtype} {run_id(run)}")
    assert torch.linalg.matrix_norm(O.double(), 2).max() < 1.3


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_many_steps_of_ordinary_rows(dtype):
    """Many steps of full rank; powers of two in front change nothing; zeros stay; a bad matrix is alone."""
    g = torch.Generator(device="cuda").manual_seed(3)
    G = torch.randn(5, 24, 500, device="cuda", generator=g).to(dtype)
    for steps, coefs in ((16, COEFS), (40, CUBIC), (64, COEFS)):
        O = b4.orth(G, steps, coefs, 0.0)
        ref, bound = orth_ref(G, steps, coefs, 0.0, split=dtype == F32)
        close(O, ref, bound, f"{steps} {dtype}")
        for e in (-60, 50):
            assert torch.equal(b4.orth(G * 2.0 ** e, steps, coefs, 0.0), O)
        bad = G.clone()
        bad[1, 3, 77] = float("nan")
        bad[3, -1, 0] = float("inf")
        bad[4] = 0
        got = b4.orth(bad, steps, coefs)
        whole = b4.orth(G, steps, coefs)
        assert got[[1, 3]].isnan().all() and (got[4] == 0).all() and torch.equal(got[[0, 2]], whole[[0, 2]])


def test_many_matrices():
    """A batch in which a matrix has one block for all of its columns, and one larger than a grid's part."""
    for B, m, n in ((700, 24, 4100), (33000, 3, 20)):
        G, Q, K = dependent(m, n, F32, "twice", B, matrices=B)
        ref = dependent_ref(Q, K, 25)
        close(b4.orth(G, 25, COEFS, 0.0), ref, 4 * narrow_bound(ref, m, 25), f"{B} of {m} x {n}")


def test_captured():
    G, Q, K = dependent(24, 1024, BF16, "twice", 1)
    ref = dependent_ref(Q, K, 25)
    eager = b4.orth(G, 25, COEFS, 0.0)
    held = torch.zeros_like(G)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O = b4.orth(held, 25, COEFS, 0.0)
    for _ in range(3):
        held.copy_(G)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, eager)
        O.fill_(float("nan"))
    close(eager, ref, narrow_bound(ref, 24, 25), "captured")


def ordinary(shape, dtype, kind, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    L, m, n = shape
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)
    if kind == "spread":
        return normal(*shape).to(dtype)
    return (torch.matmul(normal(L, m, 8) * torch.exp(-0.3 * torch.arange(8, device="cuda")), normal(L, 8, n))).to(dtype)


LARGE = [(kind, steps, coefs) for kind in ("spread", "low", "fades") for steps, coefs in ((6, COEFS), (8, COEFS), (10, COEFS), (25, CUBIC))]
LARGE += [("spread", 64, COEFS), ("spread", 60, CUBIC), ("fades", 25, COEFS), ("fades", 64, COEFS), ("fades", 12, PAIRS * 6)]


@pytest.mark.parametrize("kind,steps,coefs", LARGE, ids=[f"{k}-{run_id((s, c))}" for k, s, c in LARGE])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 150, 260), (2, 300, 140), (1, 1024, 1100)], ids=str)
def test_many_steps_of_large_matrices(shape, dtype, kind, steps, coefs):
    """No further off than the stated roundings take it: the last steps' growth is that of five usual ones."""
    if kind == "fades":
        G = fades(min(shape[1:]), max(shape[1:]), dtype, 5, 1e-6)
        G = turn(G) if shape[1] > shape[2] else G
    else:
        G = ordinary(shape, dtype, kind, 5)
    label = f"{shape} {dtype} {kind} {run_id((steps, coefs))}"
    print(label, flush=True)
    ref, bound = rounded_ref(G, steps, coefs)
    bound = bound + carried(G, steps, coefs)
    close(b4.orth(G, steps, coefs, 0.0), ref, bound, label)
    W, M = torch.zeros_like(G), torch.zeros(G.shape, device="cuda")
    b4.orth_step(W, G, M, -1.0, 0.0, False, scale=1.0, steps=steps, coefs=coefs, eps=0.0)
    close(W, ref, bound, label + " update")


def test_many_steps_in_parts():
    """A batch of which the workspace takes a part at a time: the same bits wherever a matrix stands."""
    G = ordinary((2600, 100, 300), BF16, "spread", 6)
    G[2599] = G[1300] = G[0]
    O = b4.orth(G, 8)
    ref, bound = rounded_ref(G[:1], 8, COEFS)
    close(O[:1], ref, bound, "first")
    assert torch.equal(O[0], O[1300])
    close(O[2599:], ref, bound, "last")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 24, 1000), (2, 500, 40), (1, 100, 700)], ids=str)
def test_a_steep_first_step(shape, dtype):
    """A first step that alone multiplies by more than the first run of a narrow matrix takes."""
    G = ordinary(shape, dtype, "spread", 8)
    coefs = [(1.0, 60.0, 0.0)] + [CUBIC] * 6
    ref, bound = orth_ref(G, 7, coefs, 0.0, split=dtype == F32)
    close(b4.orth(G, 7, coefs, 0.0), ref, bound, f"{shape} {dtype}")
