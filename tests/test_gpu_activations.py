"""The activations of ``imat_forward`` at the size of their own values: on the negative side they fall to nothing, and a bound of the size of
the argument sees nothing there.  The weights are zeros, so the bias is the activation's argument, exactly."""
import math

import pytest
import torch

from ff_util import TYPES, U, Filter, Plan, act64, generator, half_step, rows8, stream
from paper_2006_11735_b200 import binding as B

pytestmark = pytest.mark.gpu

FORMS = [(2, 640, "stream"), (40, 640, "few"), (100, 4096, "few"), (2100, 640, "bulk")]
FAR = [0.0, 1e-30, 1e-5, 16, 20, 40, 80, 86, 87, 87.5, 88, 88.5, 89, 95, 100, 103, 110, 200, 1e4, 1e18, 1e30, 3e38]


def _arguments():
    at = torch.cat([torch.linspace(-14.5, 14.5, 2146), torch.linspace(-106.0, -14.0, 146), torch.tensor([s * v for v in FAR for s in (1.0, -1.0)])])
    return at.cuda()                             # 2336


def own_bound(act, y, dtype):
    """(value, bound) for float arguments y (in 64 bits), of the value's size.  U is half a step of float, relative; documented errors are in steps of 2 U.

    GELU, y / 2 times e or 2 - e, e = exp(-y^2 / 2) times a polynomial of t = 1 / (1 + c |y|).  Float results: the fit 1e-8, its evaluation (t 2 steps, the sums and products
    of the last terms) 10 U, the exponential's argument U y^2 / 2, expf 2 steps, two products, the difference to 2.  16-bit results: the fit 1.7e-6, the argument
    as a base 2 exponential's (0.3 U and U of its root, twice, and U) 3.6 U y^2 / 2.
    The others, y times 1 / (1 + exp(-z)).  Float results: expf 2 steps and z's own error (z = y: none; z = y (c0 + c1 y^2): both coefficients, the square, the sum, the
    product: 4 U of it) weigh sigmoid(-z); the product with e, the sum, the reciprocal and the product with it U each.  16-bit results: 2 steps for the exponential, 1.4 U of its
    argument for the change of base, 2 steps for the reciprocal.
    The last term: what an exponential that is no normal number (float: the last place of one) may lose."""
    v, a = act64(act, y), y.abs()
    fine = dtype is torch.float32
    if act == "gelu":
        h = (y * y / 2).clamp_max(110.0)                # (beyond, erfc is 0 or 2)
        rel = 1e-8 / U + 17.1 + h if fine else 1.7e-6 / U + 17.1 + 3.6 * h
        least = a / 2
    else:
        z = y if act == "silu" else 2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)
        off = 0.0 if act == "silu" else 4.01 * z.abs()
        rel = (4 + off) * torch.sigmoid(-z) + 4.2 if fine else (4 + 1.4 * z.abs() + off) * torch.sigmoid(-z) + 7.2
        least = a
    # (where the value is nothing the factor may be anything, infinite too)
    e = torch.where(v == 0, torch.zeros_like(v), rel * U * v.abs()) + (least.clamp_max(1e4) * 4 + 1) * (2.0 ** -149 if fine else 2.0 ** -126)
    return v, e * (1 + torch.finfo(dtype).eps) + half_step(dtype, v)


def _plan(act, dtype, at, k, gated):
    gen, n = generator(0), at.numel()
    zeros = torch.zeros(n, k, device="cuda", dtype=torch.int16)
    f = Filter(gen, n, k, w=zeros)
    f.bias = at
    up = None
    if gated:
        up = Filter(gen, n, k, w=zeros)
        up.bias = torch.ones(n, device="cuda")
    return Plan(dtype, f, up, act)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("m,k,kernel", FORMS)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_at_their_own_size(act, dtype, m, k, kernel, gated):
    at = _arguments()
    plan = _plan(act, dtype, at, k, gated)
    assert plan.describe(m).startswith(kernel)
    out = plan(*rows8(generator(1), m, k))
    assert torch.equal(out, out[:1].expand_as(out))
    v, e = own_bound(act, at.double(), TYPES[dtype])
    some = v.abs() < torch.finfo(TYPES[dtype]).max
    off = (out[0].double() - v).abs()
    worst = int(torch.where(some, off / e, torch.zeros_like(off)).argmax())
    assert (off <= e)[some].all(), "%s(%g) = %g, not %g" % (act, at[worst], out[0, worst], v[worst])
    B.iconv_check(stream())


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_float_at_points_of_the_negative_side(act):
    """Two to four digits that float results had lost; by hand, apart from the bound above."""
    at = torch.tensor([-2.0, -3.0, -4.0, -5.0, -8.0, -10.0, -12.0], device="cuda")
    out = _plan(act, "f32", at, 16, False)(*rows8(generator(1), 3, 16))
    v = act64(act, at.double())
    # (the second term: what is no normal number; at -12 the value of gelu_tanh is 12 exp(-142) = 1e-61, of which float has nothing)
    assert ((out[0].double() - v).abs() <= 3e-5 * v.abs() + (4 * at.double().abs() + 1) * 2.0 ** -149).all(), ((out[0].double() - v).abs() / v.abs()).tolist()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_what_is_no_number(act, dtype):
    """As the formulas give them: infinity times nothing is no number."""
    at = torch.tensor([float("inf"), float("-inf"), float("nan"), 1.0], device="cuda")
    for m, k, _ in FORMS:
        out = _plan(act, dtype, at, k, False)(*rows8(generator(1), m, k))
        assert (out[:, 0] == float("inf")).all() and torch.isnan(out[:, 1:3]).all() and torch.isfinite(out[:, 3]).all()
