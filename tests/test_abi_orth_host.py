"""Host-side checks of the orthogonalisation and its update (no GPU needed): bad arguments return their
code before anything touches the device (the addresses are fake; every call below returns first), the
reference against closed forms, and what the binding refuses."""
import ctypes
import math

import pytest
import torch

import paper_2606_07574_amd as b4
from tests._orth import COEFS, orth_ref

OK, NULL, SIZE, DTYPE, ALIGN, OVERLAP, STEPS, EPS, WORK = 0, -1, -2, -5, -6, -7, -8, -14, -15
MB = 1 << 28
ARRAY = (ctypes.c_float * 15)(*(COEFS * 5))


def place(k):
    return (k + 1) * MB  # fake, aligned, far apart


def test_orth():
    f = b4.lib().birkhoff4_orth
    work = b4.lib().birkhoff4_orth_work(2, 30, 50, b4.F32)
    assert work > 0
    good = dict(G=place(0), dt=b4.BF16, out=place(1), o_dt=b4.F32, coefs=ARRAY, steps=5, eps=1e-7, work=place(2), size=work, B=2,
                rows=30, cols=50, stream=None)
    call = lambda **kw: f(*{**good, **kw}.values())
    assert call(B=0) == OK and call(rows=0) == OK and call(cols=0) == OK
    for k in ("B", "rows", "cols"):
        assert call(**{k: -1}) == SIZE
    assert call(rows=(1 << 20) + 1) == SIZE and call(cols=(1 << 20) + 1) == SIZE and call(B=(1 << 26) + 1) == SIZE
    assert call(rows=70000, cols=70000) == SIZE and call(B=1 << 26, rows=1 << 15, cols=1 << 15) == SIZE
    assert call(dt=2) == DTYPE and call(o_dt=-1) == DTYPE
    assert call(steps=0) == STEPS and call(steps=65) == STEPS
    for eps in (-1e-6, float("inf"), float("nan")):
        assert call(eps=eps) == EPS
    assert call(size=work - 1) == WORK and call(size=0) == WORK
    for k in ("G", "out", "coefs", "work"):
        assert call(**{k: None}) == NULL
    assert call(G=good["G"] + 1) == ALIGN and call(out=good["out"] + 2) == ALIGN and call(work=good["work"] + 8) == ALIGN
    for out, other in (("out", "G"), ("work", "G"), ("work", "out")):
        assert call(**{out: good[other]}) == OVERLAP
    assert call(out=place(0) + 2 * 30 * 50 * 2 - 4) == OVERLAP


def test_orth_step():
    f = b4.lib().birkhoff4_orth_step
    work = b4.lib().birkhoff4_orth_work(2, 50, 30, b4.BF16)
    good = dict(W=place(0), w_dt=b4.BF16, G=place(1), g_dt=b4.F32, M=place(2), momentum=0.9, nesterov=1, lr=0.1, lr_at=place(3),
                decay=0.1, scale=1.0, coefs=ARRAY, steps=5, eps=1e-7, work=place(4), size=work, B=2, rows=50, cols=30, stream=None)
    call = lambda **kw: f(*{**good, **kw}.values())
    assert call(B=0) == OK
    assert call(rows=-1) == SIZE and call(w_dt=3) == DTYPE and call(g_dt=-1) == DTYPE and call(steps=-1) == STEPS
    assert call(eps=-1.0) == EPS and call(size=work - 1) == WORK
    for k in ("W", "G", "M", "coefs", "work"):
        assert call(**{k: None}) == NULL
    for k, by in (("W", 1), ("G", 2), ("M", 2), ("lr_at", 1), ("work", 4)):
        assert call(**{k: good[k] + by}) == ALIGN
    for out in ("W", "M", "work"):
        for other in ("W", "G", "M", "lr_at", "work"):
            if other != out:
                assert call(**{out: good[other]}) == OVERLAP


def test_orth_work():
    f = b4.lib().birkhoff4_orth_work
    assert f(0, 8, 8, b4.F32) == 0 and f(3, 0, 8, b4.F32) == 0
    assert f(-1, 8, 8, b4.F32) == SIZE and f(1, 8, 8, 7) == DTYPE
    for dt in (b4.F32, b4.BF16):
        assert f(1, 4096, 4096, dt) < 24 * 4096 * 4096 + (1 << 16)
        assert f(1, 100, 7000, dt) == f(1, 7000, 100, dt)
        # a large batch goes through a bounded workspace
        assert f(1 << 20, 64, 64, dt) <= (1 << 30)


def test_reference():
    """Closed forms: a diagonal matrix's values go through the polynomial; the matrix's size does not
    matter but for eps; and the polar factor's singular vectors stay."""
    def poly(s, steps=5):
        for _ in range(steps):
            s = COEFS[0] * s + COEFS[1] * s ** 3 + COEFS[2] * s ** 5
        return s

    d = torch.tensor([3.0, 1.0, 0.25, 0.01], dtype=torch.float64)
    G = torch.zeros(1, 4, 6, dtype=torch.float64)
    G[0, range(4), range(4)] = d
    want = poly(d / d.norm())
    got, _ = orth_ref(G, eps=0.0)
    assert torch.allclose(got[0, range(4), range(4)], want, rtol=1e-12)
    assert torch.allclose(orth_ref(G * 1e3, eps=0.0)[0], got, rtol=1e-12)
    g = torch.Generator().manual_seed(1)
    G = torch.randn(2, 7, 5, generator=g, dtype=torch.float64)
    U, s, V = torch.linalg.svd(G, full_matrices=False)
    want = U @ torch.diag_embed(poly(s / torch.linalg.vector_norm(s, dim=1, keepdim=True))) @ V
    assert torch.allclose(orth_ref(G, eps=0.0)[0], want, rtol=1e-10, atol=1e-12)
    # the usual coefficients: from 0.003 on within 0.68..1.21
    s = poly(torch.linspace(0.003, 1, 100001, dtype=torch.float64))
    assert 0.68 < s.min() and s.max() < 1.21


def test_bounds_tell_mistakes():
    """One step more or less, another coefficient, a row exchanged: each is outside what roundings may do."""
    g = torch.Generator().manual_seed(2)
    G = torch.randn(2, 24, 100, generator=g)
    for split in (True, False):
        ref, bound = orth_ref(G, split=split)
        size = torch.linalg.vector_norm(ref, dim=(1, 2))
        assert (bound / size < (1e-5 if split else 0.03)).all()
        swapped = ref.clone()
        swapped[:, [3, 4]] = ref[:, [4, 3]]
        other = tuple(1.05 * c for c in COEFS)
        for wrong in (orth_ref(G, steps=4)[0], orth_ref(G, steps=6)[0], orth_ref(G, coefs=[COEFS] * 4 + [other])[0], swapped):
            assert (torch.linalg.vector_norm(wrong - ref, dim=(1, 2)) > 1.2 * bound + 2.0 ** -8 * size * (not split)).all()


def test_refusals():
    x = torch.randn(3, 8)
    for call in (lambda: b4.orth(x), lambda: b4.orth_step(x, x, x, 0.1)):
        with pytest.raises(b4.Birkhoff4Error, match="GPU"):
            call()
    for call in (lambda: b4.orth(x.requires_grad_(True)),):
        with pytest.raises(RuntimeError, match="no derivative"):
            call()
    for coefs, steps in (((1.0, 2.0), 5), (((1.0, 2.0, 3.0),) * 4, 5), (((1.0, 2.0),) * 5, 5)):
        with pytest.raises(ValueError, match="triples"):
            b4._steps(coefs, steps)
    assert list(b4._steps([[1, 2, 3], (4, 5, 6)], 2)[0]) == [1, 2, 3, 4, 5, 6]
    for steps in (0, 65):
        with pytest.raises(ValueError, match="step count"):
            b4._steps(COEFS, steps)
    assert math.isclose(b4.ORTH_COEFS[0], COEFS[0])


def test_coefficients_are_taken_by_value():
    """A coefficient that changes between calls, in a tensor that stays, is another coefficient."""
    c = torch.tensor(2.0)
    first, _ = b4._steps((c, 0.0, 0.0), 1)
    c += 1
    second, _ = b4._steps((c, 0.0, 0.0), 1)
    assert list(first) == [2.0, 0.0, 0.0] and list(second) == [3.0, 0.0, 0.0]
