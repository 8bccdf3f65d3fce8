"""Host-side checks of the layer norm (no GPU needed): bad arguments return their code before anything
touches the device (the addresses are fake; every call below returns first), the reference's gradients
against differences, and what the binding refuses."""
import pytest
import torch
from torch.autograd import forward_ad

import paper_2606_07574_amd as b4
from tests._norm import norm_back_ref, norm_ref

OK, NULL, SIZE, DTYPE, ALIGN, OVERLAP, CHANNELS, EPS, WORK = 0, -1, -2, -5, -6, -7, -13, -14, -15
MB = 1 << 28


def place(k):
    return (k + 1) * MB  # fake, aligned, far apart


def test_norm_fwd():
    f = b4.lib().birkhoff4_norm_fwd
    good = dict(X=place(0), dt=b4.BF16, weight=place(1), bias=place(2), w_dt=b4.F32, eps=1e-5, Y=place(3), mean=place(4),
                rstd=place(5), B=10, C=65, stream=None)
    call = lambda **kw: f(*{**good, **kw}.values())
    assert call(B=0) == OK and call(B=0, X=None, Y=None) == OK
    assert call(B=-1) == SIZE and call(B=(1 << 31) + 1) == SIZE and call(C=(1 << 20) + 1) == SIZE
    assert call(B=1 << 31, C=1 << 20) == SIZE
    assert call(dt=2) == DTYPE and call(w_dt=-1) == DTYPE
    assert call(C=0) == CHANNELS and call(C=-8) == CHANNELS
    for eps in (-1e-6, float("inf"), float("nan")):
        assert call(eps=eps) == EPS
    for k in ("X", "Y"):
        assert call(**{k: None}) == NULL
    for k in ("X", "weight", "bias", "Y", "mean", "rstd"):
        assert call(**{k: good[k] + 8}) == ALIGN
    for out in ("Y", "mean", "rstd"):
        for other in ("X", "weight", "bias", "Y", "mean", "rstd"):
            if other != out:
                assert call(**{out: good[other]}) == OVERLAP
    # the last value counts: ten rows of 65 two-byte values are 1300 bytes
    assert call(Y=place(0) + 1296) == OVERLAP


def test_norm_bwd():
    f = b4.lib().birkhoff4_norm_bwd
    work = b4.lib().birkhoff4_norm_work(10, 65, b4.F32)
    names = ("X", "dt", "weight", "w_dt", "mean", "rstd", "dY", "dX", "dweight", "dbias", "work")
    good = {k: place(i) for i, k in enumerate(names)}
    good.update(dt=b4.F32, w_dt=b4.BF16, size=work, B=10, C=65, stream=None)
    call = lambda **kw: f(*{**good, **kw}.values())
    assert call(B=-1) == SIZE and call(dt=-1) == DTYPE and call(w_dt=5) == DTYPE and call(C=0) == CHANNELS
    assert call(size=work - 1) == WORK and call(size=0) == WORK
    for k in ("X", "mean", "rstd", "dY", "work"):
        assert call(**{k: None}) == NULL
    for k in names:
        if k not in ("dt", "w_dt"):
            assert call(**{k: good[k] + 4}) == ALIGN
    for out in ("dX", "dweight", "dbias", "work"):
        for other in names:
            if other not in (out, "dt", "w_dt"):
                assert call(**{out: good[other]}) == OVERLAP
    # nothing asked for
    assert call(dX=None, dweight=None, dbias=None, work=None, size=0) == OK
    assert call(B=0, dweight=None, dbias=None) == OK


def test_norm_work():
    f = b4.lib().birkhoff4_norm_work
    assert f(0, 64, b4.F32) == 0 and f(-1, 64, b4.F32) == SIZE and f(5, 0, b4.F32) == CHANNELS and f(5, 64, 9) == DTYPE
    for C in (1, 8192, 8193, 1 << 20):
        for dt in (b4.F32, b4.BF16):
            assert f(1, C, dt) == 8 * C and 8 * C <= f(100000, C, dt) <= 256 * 8 * C + (1 << 24)
    # a few per cent of the rows for a training batch
    assert f(32768, 4096, b4.BF16) < 0.05 * 32768 * 4096 * 2


def test_reference_against_differences():
    """The formula's gradients in float64 against central differences."""
    g = torch.Generator().manual_seed(3)
    x, w, b, dy = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((3, 7), (7,), (7,), (3, 7)))
    grads = norm_back_ref(norm_ref(x, w, b, 1e-3)[2], dy)[0]
    value = lambda: (norm_ref(x, w, b, 1e-3)[0][0] * dy).sum()
    for t, grad in zip((x, w, b), grads):
        for i in range(t.numel()):
            at, h = t.view(-1), 1e-5
            was = at[i].item()
            at[i] = was + h
            up = value()
            at[i] = was - h
            down = value()
            at[i] = was
            # the third derivative's h^2 and two roundings of a value of order ten over 2 h
            assert abs((up - down).item() / (2 * h) - grad.reshape(-1)[i].item()) < 1e-8


def test_refusals():
    x = torch.randn(3, 8)
    for call in (lambda: b4.norm_fwd(x), lambda: b4.norm(x), lambda: b4.norm_bwd(x, None, x[:, 0], x[:, 0], x)):
        with pytest.raises(b4.Birkhoff4Error, match="GPU"):
            call()


@pytest.mark.parametrize("which", [0, 1, 2])
def test_tangents_are_refused(which, monkeypatch):
    monkeypatch.setattr(b4, "_normed", lambda x, *rest: (3, 8, 0))
    monkeypatch.setattr(b4, "_norm_fwd", lambda x, *rest: (x, x[:, 0], x[:, 0]))
    args = [torch.randn(3, 8), torch.randn(8), torch.randn(8)]
    with forward_ad.dual_level():
        args[which] = forward_ad.make_dual(args[which], torch.ones_like(args[which]))
        with pytest.raises(NotImplementedError, match="jvp"):
            b4.norm(*args)
