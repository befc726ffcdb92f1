"""The gated block where the gate is far negative: GELU's values there are small, and have to be good to their own size.  The
weights pick one value of x as the gate and one as the other factor, so that both are exact."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import operator_forms as forms  # noqa: E402

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def tf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_32479_amd as tf
    return tf


@pytest.mark.parametrize("dtype", [BF16, FP32, FP16])
@pytest.mark.parametrize("rows", [40, 700])   # weights streamed to registers; tiles
def test_gelu_of_far_negative_gates(tf, dtype, rows):
    # fp16's smallest normal value is 6e-5: there the other factor is large, and the gate not as far out
    least, factor = (-5.0, 30000.0) if dtype == FP16 else (-8.0, 3.0)
    a = torch.linspace(least, -2.5, rows).to(dtype)
    x = torch.zeros(rows, 8, dtype=dtype)
    x[:, 0], x[:, 1] = a, factor
    w = torch.zeros(2, 1, 8, dtype=dtype)
    w[0, 0, 0] = w[1, 0, 1] = 1.0
    d_out = torch.full((rows, 1), 0.75, dtype=dtype)
    c = [t.cuda() for t in (x, w[0], w[1])]
    A = a.double()
    phi, der = 0.5 * torch.erfc(-A / math.sqrt(2.0)), torch.exp(-A * A / 2) / math.sqrt(2 * math.pi)
    # One rounding to the type (its half step); the function: an exponential of up to 46 in base 2, whose argument's roundings
    # (two of 2^-24 of 46 ln 2) and own (2^-22) make 2^-18, and a few roundings of 2^-24; the derivative phi(a) a + Phi(a), which
    # is a fifth smaller than its larger term, half as much again
    tol = forms.HALF[dtype] + 2.0 ** -17
    h = tf.gated_ffn(*c, activation="gelu")[:, 0].double().cpu()
    assert ((h / (A * phi * float(x[0, 1])) - 1).abs().max().item()) <= tol
    dx = tf.gated_ffn_backward(d_out.cuda(), *c, activation="gelu")[0].double().cpu()
    for got, want in ((dx[:, 0], 0.75 * float(x[0, 1]) * (phi + A * der)), (dx[:, 1], 0.75 * A * phi)):
        fine = want.abs() >= torch.finfo(dtype).tiny
        assert bool(fine.any()) and ((got / want - 1).abs()[fine].max().item()) <= 1.5 * tol
