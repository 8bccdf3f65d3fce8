"""Host-side checks of the streams' read and write (no GPU needed): bad arguments return their code
before anything touches the device. The addresses are fake; every call below returns first."""
import pytest

import paper_2606_07574_amd as b4

OK, NULL, SIZE, DTYPE, ALIGN, OVERLAP, CHANNELS, EPS, WORK, DROP = 0, -1, -2, -5, -6, -7, -13, -14, -15, -16
MB = 1 << 28


def place(k):
    return (k + 1) * MB  # fake, aligned, far apart


@pytest.mark.parametrize("n", [4, 8])
def test_pre_fwd(n):
    f = getattr(b4.lib(), f"birkhoff{n}_pre_fwd")
    work = getattr(b4.lib(), f"birkhoff{n}_pre_work")(10, 64, b4.BF16, 0)
    assert work > 0
    good = dict(X=place(0), W=place(1), dt=b4.BF16, alpha=place(2), bias=place(3), eps=1e-6, U=place(4), h=place(5),
                H=place(6), q=place(7), rms=place(8), work=place(9), size=work, B=10, C=64, stream=None)
    call = lambda **kw: f(*{**good, **kw}.values())
    assert call(B=0) == OK
    assert call(B=-1) == SIZE and call(B=(1 << 26) + 1) == SIZE and call(C=(1 << 24) + 8) == SIZE
    assert call(dt=2) == DTYPE
    assert call(C=0) == CHANNELS and call(C=-8) == CHANNELS and call(C=12) == CHANNELS and call(C=6, dt=b4.F32) == CHANNELS
    for eps in (-1e-6, float("inf"), float("nan")):
        assert call(eps=eps) == EPS
    assert call(size=work - 1) == WORK and call(size=0) == WORK
    for k in ("X", "W", "alpha", "bias", "U", "h", "H", "q", "rms", "work"):
        assert call(**{k: None}) == NULL
        assert call(**{k: good[k] + 8}) == ALIGN
    for out in ("U", "h", "H", "q", "rms", "work"):
        for other in ("X", "W", "alpha", "bias", "U", "h", "H", "q", "rms", "work"):
            if other != out:
                assert call(**{out: good[other]}) == OVERLAP
    # the last bytes count: U right behind X's ten tokens does not overlap it, 16 bytes earlier does
    assert call(U=place(0) + 10 * n * 64 * 2 - 16) == OVERLAP


@pytest.mark.parametrize("n", [4, 8])
def test_pre_bwd(n):
    f = getattr(b4.lib(), f"birkhoff{n}_pre_bwd")
    work = getattr(b4.lib(), f"birkhoff{n}_pre_work")(10, 64, b4.F32, 1)
    names = ("X", "W", "dt", "alpha", "bias", "q", "rms", "dU", "dh", "dH", "E", "dX", "dW", "dalpha", "dbias", "work")
    good = {k: place(i) for i, k in enumerate(names)}
    good.update(dt=b4.F32, size=work, B=10, C=64, stream=None)
    call = lambda **kw: f(*{**good, **kw}.values())
    assert call(B=-1) == SIZE and call(B=(1 << 26) + 1) == SIZE and call(dt=-1) == DTYPE and call(C=62) == CHANNELS
    assert call(C=0) == CHANNELS and call(size=work - 1) == WORK
    for k in names:
        if k == "dt":
            continue
        if k not in ("dU", "dh", "dH", "E"):
            assert call(**{k: None}) == NULL
        assert call(**{k: good[k] + 4}) == ALIGN
    for k in ("dW", "dalpha", "dbias"):
        assert call(**{k: None}, B=0) == NULL  # the sums are written without tokens too
    for out in ("dX", "dW", "dalpha", "dbias", "work"):
        for other in names:
            if other not in (out, "dt"):
                assert call(**{out: good[other]}) == OVERLAP


def test_pre_work():
    for n in (4, 8):
        f = getattr(b4.lib(), f"birkhoff{n}_pre_work")
        for backward in (0, 1):
            assert f(0, 64, b4.F32, backward) == 0
            assert f(-1, 64, b4.F32, backward) == SIZE and f(5, 0, b4.F32, backward) == CHANNELS
            assert f(5, 64, 9, backward) == DTYPE
            # a few per cent of the streams for a training batch
            assert 0 < f(32768, 4096, b4.BF16, backward) < 0.15 * 32768 * n * 4096 * 2


def test_strerror():
    texts = {b4.lib().birkhoff4_strerror(k) for k in (EPS, WORK, DROP)}
    assert len(texts) == 3 and b"unknown error" not in texts
