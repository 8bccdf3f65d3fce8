"""Forward-mode derivatives of the streams' read and write (no GPU needed: the kernels' calls are
replaced). There are none, so an input with a tangent is refused, as the residual mixing refuses it;
outputs without a tangent would be taken for a derivative of zero."""
import pytest
import torch
from torch.autograd import forward_ad

import paper_2606_07574_amd as b4

B, N, C = 3, 4, 8
R = N * N + 2 * N
calls = []


@pytest.fixture(autouse=True)
def no_kernels(monkeypatch):
    def pre_fwd(X, W, alpha, bias, eps):
        calls.append("pre")
        return torch.zeros(B, C), torch.zeros(B, N), torch.zeros(B, N, N), torch.zeros(B, R), torch.zeros(B)

    def post_fwd(H, X, h, Z, *rest):
        calls.append("post")
        return torch.zeros(B, N, C), torch.zeros(B, N, N), None, None

    def mix_fwd(n, H, X, *rest):
        return torch.zeros(B, N, C), torch.zeros(B, N, N), None, None

    monkeypatch.setattr(b4, "pre_fwd", pre_fwd)
    monkeypatch.setattr(b4, "post_fwd", post_fwd)
    monkeypatch.setattr(b4, "_mix_fwd", mix_fwd)
    calls.clear()


READ = [(B, N, C), (R, N * C), (3,), (R,)]
WRITE = [(B, N, N), (B, N, C), (B, N), (B, C)]
OPS = [("pre", b4.pre, READ), ("post", b4.post, WRITE), ("connect", lambda *a: b4.connect(*a, lambda U: U), READ),
       ("mix", b4.mix, WRITE[:2])]


@pytest.mark.parametrize("grad", ["no_grad", "none", "others"])
@pytest.mark.parametrize("name,op,shapes", OPS, ids=[o[0] for o in OPS])
def test_tangents_are_refused(name, op, shapes, grad):
    for k in range(len(shapes)):
        with forward_ad.dual_level():
            args = [torch.randn(s, requires_grad=grad == "others" and i != k) for i, s in enumerate(shapes)]
            args[k] = forward_ad.make_dual(args[k], torch.ones(shapes[k]))
            with torch.set_grad_enabled(grad != "no_grad"):
                with pytest.raises(NotImplementedError, match="jvp"):
                    op(*args)


@pytest.mark.parametrize("name,op,shapes", OPS[:3], ids=[o[0] for o in OPS[:3]])
def test_branch_tangent_is_refused(name, op, shapes):
    """Under torch.func.jvp, and where the tangent comes from the branch alone."""
    args = [torch.randn(s) for s in shapes]
    with pytest.raises(RuntimeError):
        torch.func.jvp(lambda x: op(x, *args[1:]), (args[0],), (torch.ones(shapes[0]),))
    with forward_ad.dual_level(), pytest.raises(NotImplementedError, match="jvp"):
        weight = forward_ad.make_dual(torch.ones(C), torch.ones(C))
        b4.connect(*(torch.randn(s) for s in READ), lambda U: U * weight)


def test_no_tangents():
    """A level without tangents among the inputs changes nothing, and without gradients the calls
    go straight to the kernels."""
    for level in (False, True):
        args = [torch.randn(s) for s in READ]
        if level:
            with forward_ad.dual_level():
                Y = b4.connect(*args, lambda U: U)
        else:
            Y = b4.connect(*args, lambda U: U)
        assert Y.shape == (B, N, C) and not Y.requires_grad
    assert calls == ["pre", "post"] * 2
