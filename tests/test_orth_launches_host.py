"""Which forms of the orthogonalisation's kernels are launched, as the host decides it (no GPU needed): the sizes of the
GPU tests run all of them."""
import paper_2606_07574_amd as b4
from tests._launches import kernels, launches
from tests._orth import COEFS
from tests._orth_tiles import BF16, F32, ORTH, STEP
from tests.test_gpu_orth import SIZES

AT = 1 << 42  # fake addresses, far apart
ROOM = 1 << 41


def code(dtype):
    return b4.BF16 if dtype == BF16 else b4.F32


def orth(B, m, n, g, o, steps=5, coefs=COEFS):
    return ("birkhoff4_orth", "pipicifpllllp", [AT, code(g), 2 * AT, code(o), list(coefs) * steps, steps, 1e-7, 3 * AT, ROOM, B, m, n, None])


def step(B, m, n, w, g, steps=5):
    return ("birkhoff4_orth_step", "pipipfifpffcifpllllp",
            [AT, code(w), 2 * AT, code(g), 3 * AT, 0.9, 1, 0.1, None, 0.0, 1.0, list(COEFS) * steps, steps, 1e-7, 4 * AT, ROOM, B, m, n, None])


def test_every_product_is_run(tmp_path):
    calls = [orth(*s, t, t, k) for s, t, k in ORTH] + [step(*s, t, t, k) for s, t, k in STEP]
    found = launches(calls, tmp_path)
    assert all(c == 0 for c, _ in found)
    run = {k[:2] for _, launched in found for k in launched}
    there = {k for k in kernels(tmp_path) if k[0] == "orth_product_kernel"}
    assert len(there) > 40 and there == {k for k in run if k[0] == "orth_product_kernel"}, sorted(there - run)


def test_every_kernel_is_run(tmp_path):
    """The others: narrow ones of every number of tiles, of both types in and out, few steps and many."""
    calls = []
    for m in (3, 20, 40, 64, 80, 100):
        for shape in ((2, m, 200), (2, 200, m)):
            for t in (F32, BF16):
                for u in (F32, BF16):
                    for steps in (5, 8):
                        calls += [orth(*shape, t, u, steps), step(*shape, t, u, steps)]
    calls += [orth(*s, t, t, k) for s, t, k in ORTH] + [step(*s, t, t, k) for s, t, k in STEP]
    calls += [orth(*((1,) * (3 - len(s)) + tuple(s)), F32, F32) for s in SIZES]
    run = {k[:2] for _, launched in launches(calls, tmp_path) for k in launched}
    there = {k for k in kernels(tmp_path) if k[0].startswith("orth_")}
    assert there == run, sorted(there - run)


def test_many_steps(tmp_path):
    """Runs of a narrow matrix: one for steps that multiply to 512 at most, two for more, one from the start where the first
    step alone is more than the first run takes."""
    run = lambda *call: [k[0] for k in launches([orth(1, 24, 64, F32, F32, *call)], tmp_path)[0][1]]
    few, many = ["orth_narrow_gram_kernel", "orth_narrow_poly_kernel"], ["orth_narrow_again_kernel", "orth_narrow_poly_kernel"]
    assert run(5) == few + ["orth_narrow_apply_kernel"]
    assert run(6) == few + many + ["orth_narrow_apply_kernel"]
    assert run(1, (1.0, 600.0, 0.0)) == few + ["orth_narrow_apply_kernel"]
    cubic = (1.5, -0.5, 0.0)
    assert run(15, cubic) == few + ["orth_narrow_apply_kernel"] and run(16, cubic) == few + many + ["orth_narrow_apply_kernel"]
