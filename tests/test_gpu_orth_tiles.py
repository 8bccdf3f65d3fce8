"""GPU parity of every form of the orthogonalisation's product kernel with float64, tile by tile."""
import pytest
import torch

import paper_2606_07574_amd as b4
from tests._orth import close, orth_ref, turn
from tests._orth_tiles import BF16, F32, ORTH, STEP, close_tiles

pytestmark = pytest.mark.gpu


def spread(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=g).to(dtype)


@pytest.mark.parametrize("shape,dtype,steps", ORTH, ids=str)
def test_products(shape, dtype, steps):
    G = spread(shape, dtype, sum(shape))
    print(shape, dtype, steps, flush=True)
    close_tiles(b4.orth(G, steps), G, steps, "wide")
    close_tiles(turn(b4.orth(turn(G), steps)), G, steps, "tall")


@pytest.mark.parametrize("shape,dtype,steps", STEP, ids=str)
def test_products_of_updates(shape, dtype, steps):
    """Steps without X, which may be off by 1.6 times what the others are."""
    G = spread(shape, dtype, sum(shape))
    print(shape, dtype, steps, flush=True)
    for tall in (False, True):
        D = turn(G) if tall else G
        W, M = torch.zeros_like(D), torch.zeros_like(D)
        b4.orth_step(W, D, M, -1.0, 0.0, False, scale=1.0, steps=steps)
        close_tiles(turn(W) if tall else W, G, steps, "tall" if tall else "wide", 1.6)


@pytest.mark.parametrize("shape,dtype", [((14, 723, 723), BF16), ((1, 1326, 1707), BF16), ((1, 580, 3330), F32), ((52, 140, 524), F32)], ids=str)
def test_updated_weights(shape, dtype):
    """The update that a product ends with: what it reads of the weights is what it writes to."""
    G, W, M = spread(shape, dtype, 1), spread(shape, dtype, 2), torch.zeros(shape, device="cuda")
    held = torch.zeros_like(G)  # the direction, in the weights' type
    b4.orth_step(held, G, torch.zeros_like(M), -1.0, 0.0, False, scale=1.0)
    got = W.clone()
    b4.orth_step(got, G, M, 0.25, 0.0, False, decay=0.5, scale=1.0)
    want = W.double() * (1 - 0.25 * 0.5) - 0.25 * held.double()
    if dtype == F32:
        # the product with the rate and the sum are rounded once each, as is the shrunk weight
        bound = 3 * 2.0 ** -24 * (W.double().abs() + held.double().abs())
    else:
        bound = 1.01 * 2.0 ** -8 * (0.25 * held.double().abs() + want.abs())  # held is rounded as the result is
    assert ((got.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("m", [3, 20, 40, 64, 80, 100])
@pytest.mark.parametrize("types", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)], ids=["f32", "f32bf16", "bf16f32", "bf16"])
@pytest.mark.parametrize("steps", [5, 8])
def test_types(m, types, steps):
    """Every number of tiles of a narrow matrix, both types in and out; an update from either into either."""
    kind, result = types
    code = lambda t: b4.BF16 if t == BF16 else b4.F32
    for shape in ((2, m, 200), (2, 200, m)):
        G = spread(shape, kind, m + steps)
        out, lib = torch.empty(shape, dtype=result, device="cuda"), b4.lib()
        size = lib.birkhoff4_orth_work(*shape, code(result))
        work = torch.empty(size, dtype=torch.uint8, device="cuda")
        array, _ = b4._steps(b4.ORTH_COEFS, steps)
        assert lib.birkhoff4_orth(G.data_ptr(), code(kind), out.data_ptr(), code(result), array, steps, 1e-7, work.data_ptr(), size,
                                  *shape, torch.cuda.current_stream().cuda_stream) == 0
        # eight steps of bf16 results: the last five of one piece, where the side is more than 80
        ref, bound = orth_ref(G, steps, split=result == F32 or (steps > 5 and m <= 80))
        close(out, ref, bound, f"{shape} {types} {steps}")
        W, M = torch.zeros(shape, dtype=result, device="cuda"), torch.zeros(shape, device="cuda")
        b4.orth_step(W, G, M, -1.0, 0.0, True, scale=1.0, steps=steps)
        close(W, ref, bound, f"{shape} {types} {steps} update")
