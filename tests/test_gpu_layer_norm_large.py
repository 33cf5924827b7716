"""Large layer norms, whose rows are read in other chunks than small ones' where they lie on 16-byte borders: the same bits wherever rows lie, and
the backward pass's sums over all rows, exactly."""
import pytest
import torch

from paper_2602_08923_amd import binding as B
from tests import plain_activations as P

pytestmark = pytest.mark.gpu

# every way that rows are kept: 16, 32, 64, 128, 256 and 512 threads to a row, one to four chunks each, and rows beyond
WIDTHS = [128, 97, 250, 500, 1000, 1029, 2048, 3000, 4096, 5000, 6151, 8192, 9001, 12300, 16384, 17000]


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield torch.device("cuda:0")
    torch.cuda.empty_cache()


def rows_of(cols, dtype):
    """So many that x alone has 128 MiB, with a turn of the blocks that is not full."""
    return (1 << 27) // (cols * dtype.itemsize) + 5


def wide(rows, cols, ld, dtype, dev):
    return torch.empty(rows, ld, dtype=dtype, device=dev)[:, :cols]


@pytest.mark.parametrize("cols", WIDTHS)
def test_the_same_bits_wherever_rows_lie(dev, cols):
    """fp32 rows on 16-byte borders, rows of which every other one is off them, and one operand of each."""
    rows = rows_of(cols, torch.float32)
    g = torch.Generator(device=dev).manual_seed(cols)
    even, odd = cols + -cols % 4, cols + -cols % 4 + 1
    x, dy = wide(rows, cols, even, torch.float32, dev), wide(rows, cols, even, torch.float32, dev)
    x.copy_(torch.randn(rows, cols, generator=g, device=dev) + 0.3)
    dy.copy_(torch.randn(rows, cols, generator=g, device=dev))
    x2, dy2, out = [wide(rows, cols, odd, torch.float32, dev) for _ in range(3)]
    x2.copy_(x)
    dy2.copy_(dy)
    weight, bias = torch.linspace(0.5, 1.5, cols, device=dev), torch.linspace(-1, 1, cols, device=dev)
    room = wide(rows, cols, even, torch.float32, dev)
    y, saved = B.dq_layer_norm(x, weight, bias, save=True, out=room)
    for a, o in ((x2, out), (x, out), (x2, wide(rows, cols, even, torch.float32, dev))):
        y2, s2 = B.dq_layer_norm(a, weight, bias, save=True, out=o)
        assert bool((y2 == y).all()) and bool((s2.mean == saved.mean).all()) and bool((s2.rstd == saved.rstd).all())
    del y2, s2
    want = B.dq_layer_norm_grad(dy, saved, weight, out=room)
    for a, o in ((dy2, out), (dy, out), (dy2, wide(rows, cols, even, torch.float32, dev))):
        for got, v in zip(B.dq_layer_norm_grad(a, saved, weight, out=o), want):
            assert bool((got == v).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", WIDTHS)
def test_sums_over_all_rows_are_exact(dev, cols, dtype):
    """Small whole numbers under statistics of zero and one: n is x, every product and sum is a whole number below 2^24."""
    rows = rows_of(cols, dtype)
    g = torch.Generator(device=dev).manual_seed(cols + 1)
    ld = cols + -cols % 8
    x, dy = wide(rows, cols, ld, dtype, dev), wide(rows, cols, ld, dtype, dev)
    x.copy_(torch.randint(-3, 4, (rows, cols), generator=g, device=dev, dtype=torch.int8))
    dy.copy_(torch.randint(-3, 4, (rows, cols), generator=g, device=dev, dtype=torch.int8))
    assert 9 * rows < 2 ** 24
    saved = B.SavedNorm(B.dq_ckpt_save(x), torch.zeros(rows, device=dev), torch.ones(rows, device=dev))
    ones = torch.ones(cols, device=dev)
    dx, dw, db = B.dq_layer_norm_grad(dy, saved, ones, out=wide(rows, cols, ld, dtype, dev))
    assert bool((db.double() == dy.sum(0, dtype=torch.float64)).all())
    assert bool((dw.double() == sum((a.double() * b.double()).sum(0) for a, b in zip(x.split(16384), dy.split(16384)))).all())
    for at in range(0, rows, max(1, rows // 8)):         # dx, in parts of 64 bits' size
        k = slice(at, min(rows, at + (1 << 21) // cols))
        want = P.layer_norm_grad(dy[k], x[k], saved.mean[k], saved.rstd[k], ones)[0]
        bound = P.layer_norm_grad_bounds(dy[k], x[k], saved.mean[k], saved.rstd[k], ones, dtype, torch.float32)[0]
        assert bool(((dx[k].double() - want).abs() <= bound).all())
