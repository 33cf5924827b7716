"""How near the activations come to their formulas in binary32, over dense ranges: in half steps of binary32 (2^-24 of the value).

The hardware's exponential was off by 1.42 half steps at most, 0.58 in the mean square over an octave, its reciprocal by 1.53 and 0.48, over
all binary32 numbers of 26 octaves each; other operations round by one at most, 1 / sqrt 3 in the mean square."""
import pytest
import torch

from paper_2602_08923_amd import binding as B
from tests import plain_activations as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def between(lo, hi, dev):
    """2^18 numbers of binary32 from lo to hi, the ends left out."""
    return torch.linspace(lo, hi, 2 ** 18 + 2, dtype=torch.float64, device=dev)[1:-1].float()


def mean_square(x):
    return float(x.square().mean().sqrt())


@pytest.mark.parametrize("lo,hi", [(-1e-3, 0.0), (-0.1, -1e-3), (-1.0, -0.1), (-2.0, -1.0)])
def test_gelu_left_of_zero(dev, lo, hi):
    """z Phi(z), Phi = E t P(t), E = e^(-z^2 / 2) a square, t = 1 / (1 + 0.3 |z| / sqrt 2).  In the mean square: E twice its root's 0.58
    and a rounding; its argument's two roundings and constant, 1.4 z^2 / 2 at most; t a rounding and the reciprocal's, 0.75 together, which
    count 3.8 times in Phi (the logarithm of erfcx by that of t, at zero, where it is largest), 2.9; P's last few additions 1; the fit 0.8; three
    products 1.0.  Together 3.7 and 0.7 z^2."""
    z = between(lo, hi, dev)
    want = P.activation(z, "gelu")[0]
    off = (B.dq_gate(z, kind="gelu").double() / want - 1) / P.U
    assert mean_square(off) < 3.7 + 0.7 * lo * lo, mean_square(off)


@pytest.mark.parametrize("lo,hi", [(-1.0, -0.1), (-0.1, 0.0), (0.0, 0.1), (0.1, 1.0)])
def test_gelu_near_zero(dev, lo, hi):
    """Phi = 0.5 + z Q(z^2): the fit and its coefficients 0.9 half steps of Q, its last addition 1, what is before counts a sixth, 0.4; the
    addition of 0.5 one of Phi, the product with z one: at most."""
    z = between(lo, hi, dev)
    want = P.activation(z, "gelu")[0]
    phi = want / z.double()
    off = (B.dq_gate(z, kind="gelu").double() / want - 1).abs() / P.U
    assert bool((off < 2.05 + 2.35 * (phi - 0.5).abs() / phi).all()), float(off.max())


@pytest.mark.parametrize("lo,hi", [(-80.0, -40.0), (-40.0, -8.0), (-8.0, -1.0), (-1.0, 0.0), (0.0, 1.0), (1.0, 80.0)])
def test_silu(dev, lo, hi):
    """z / (1 + e^-z): the exponential 1.42 half steps, the sum 1, the reciprocal 1.53, what the exponent's rounding is made up for with 1, the
    product 1, at most; less than 0.1 of second order."""
    z = between(lo, hi, dev)
    want = P.activation(z, "silu")[0]
    off = (B.dq_gate(z, kind="silu").double() / want - 1) / P.U
    assert float(off.abs().max()) < 6.05, float(off.abs().max())


def test_silu_keeps_infinities_and_far_values(dev):
    z = torch.tensor([float("inf"), float("nan"), 3e38, 100.5, -100.5, -3e38, torch.finfo(torch.float32).min, 88.5, -104.0], device=dev)
    h = B.dq_gate(z, kind="silu")
    assert float(h[0]) == float("inf") and bool(torch.isnan(h[1])) and torch.equal(h[[2, 3, 7]], z[[2, 3, 7]]) and not h[[4, 5, 6, 8]].any()


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_gradients_where_the_derivative_is_zero(dev, dtype, kind):
    """dz = dh act'(z) u with dh u past the largest number: zero where act'(z) is, infinite where it is one."""
    one = torch.ones(2, 32, device=dev)
    z = torch.tensor([[-224.0], [224.0]], device=dev) * one
    _, saved = B.dq_gate(z.to(dtype), (one * 2.0 ** 70).to(dtype), kind, save=True)
    dz, du = B.dq_gate_grad((one * 2.0 ** 70).to(dtype), saved)
    assert bool((dz[0] == 0).all()) and bool((dz[1] == float("inf")).all()) and bool((du[0] == 0).all()) and bool((du[1] == 224 * 2.0 ** 70).all())
