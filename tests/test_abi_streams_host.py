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


@pytest.mark.parametrize("n", [4, 8])
def test_post_fwd(n):
    f = getattr(b4.lib(), f"birkhoff{n}_post_fwd")
    good = dict(H=place(0), h_dt=b4.F32, X=place(1), h=place(2), Z=place(3), dt=b4.BF16, p=0.1, rng=place(4), Y=place(5),
                P=place(6), dual=place(7), iters=place(8), B=10, C=64, tol=1e-6, max_iter=20, stream=None)
    call = lambda **kw: f(*{**good, **kw}.values())
    assert call(B=0) == OK
    assert call(B=-1) == SIZE and call(h_dt=3) == DTYPE and call(dt=-1) == DTYPE
    assert call(C=-8) == CHANNELS and call(C=12) == CHANNELS
    assert call(tol=-1.0) == -3 and call(max_iter=-1) == -4 and call(max_iter=10001) == -4
    for p in (1.0, -0.5, float("nan"), float("inf")):
        assert call(p=p) == DROP
    for k in ("H", "X", "h", "Z", "rng", "Y", "P"):
        assert call(**{k: None}) == NULL
    for k in ("H", "X", "h", "Z", "rng", "Y", "P", "dual", "iters"):
        assert call(**{k: good[k] + 8}) == ALIGN
    for out in ("Y", "P", "dual", "iters"):
        for other in ("H", "X", "h", "Z", "rng", "Y", "P", "dual", "iters"):
            if other != out:
                assert call(**{out: good[other]}) == OVERLAP


@pytest.mark.parametrize("n", [4, 8])
def test_post_bwd(n):
    f = getattr(b4.lib(), f"birkhoff{n}_post_bwd")
    names = ["P", "X", "h", "Z", "dY", "dt", "p", "rng", "dX", "dZ", "dh"] + (["dP"] if n == 8 else []) + ["dH"]
    good = {k: place(i) for i, k in enumerate(names)}
    good.update(dt=b4.F32, p=0.1, dh_dt=b4.F32, B=10, C=64, stream=None)
    call = lambda **kw: f(*{**good, **kw}.values())
    assert call(B=0) == OK
    assert call(B=-1) == SIZE and call(dt=2) == DTYPE and call(dh_dt=2) == DTYPE and call(C=2) == CHANNELS and call(p=1.0) == DROP
    pointers = [k for k in names if k not in ("dt", "p")]
    for k in pointers:
        assert call(**{k: None}) == NULL
        assert call(**{k: good[k] + 4}) == ALIGN
    outs = [k for k in ("dX", "dZ", "dh", "dP", "dH") if k in names]
    for out in outs:
        for other in pointers:
            # with eight streams an fp32 dH may be dP's own memory
            if other != out and {out, other} != {"dP", "dH"}:
                assert call(**{out: good[other]}) == OVERLAP
    if n == 8:
        assert call(dP=good["dH"], dh_dt=b4.BF16) == OVERLAP


def test_philox_reference():
    """The generator's reference, against the published known answers of Philox 4x32-10."""
    from tests._streams import philox
    f = 0xFFFFFFFF
    assert philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert philox((f, f, f, f), (f, f)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == \
        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_widest_rows():
    """C up to 2^20, in every call."""
    for n in (4, 8):
        work = getattr(b4.lib(), f"birkhoff{n}_pre_work")
        for dt, e in ((b4.BF16, 8), (b4.F32, 4)):
            for backward in (0, 1):
                assert work(3, 1 << 20, dt, backward) > 0 and work(3, (1 << 20) + e, dt, backward) == SIZE
                assert work(1 << 26, 64, dt, backward) > 0 and work((1 << 26) + 1, 64, dt, backward) == SIZE
