"""The activation operators where offsets pass 32 bits and where blocks take more than one turn: the far ends of large tensors against the
formulas (tests/plain_activations.py)."""
import pytest
import torch

from paper_2602_08923_amd import binding as B
from tests import plain_activations as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield torch.device("cuda:0")
    torch.cuda.empty_cache()


def fill(rows, cols, dev, seed):
    """bf16 values in large pieces (a generator's call on so many at once is slow)."""
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=dev)
    one = torch.randn(1 << 24, generator=g, device=dev).to(torch.bfloat16)
    flat = x.view(-1)
    for k, part in enumerate(flat.split(1 << 24)):
        part.copy_(one[:part.numel()] if k % 2 else one[:part.numel()].flip(0))
    return x


@pytest.mark.parametrize("rows,cols", [(70000, 32800), (70003, 32771)])
def test_checkpoints_past_2_to_the_31_entries(dev, rows, cols):
    x = fill(rows, cols, dev, 1)
    assert x.numel() > 2 ** 31
    ck = B.dq_ckpt_save(x)
    pitch = (cols + 31) // 32 * 32
    some = torch.tensor([0, 1, 65535, 65536, rows // 2, rows - 2, rows - 1], device=dev)
    codes, scales, values = P.ckpt_fields(x[some])
    data = ck.data
    assert torch.equal(data[:rows * pitch].view(rows, pitch)[some].cpu(), codes)
    assert torch.equal(data[rows * pitch:].view(rows, pitch // 32)[some].cpu(), scales)
    del x
    assert torch.equal(B.dq_ckpt_load(ck, torch.bfloat16)[some].double(), values)


def test_gates_past_2_to_the_31_entries(dev):
    rows, cols = 70000, 15500
    both = fill(rows, 2 * cols, dev, 2)
    assert both.numel() > 2 ** 31
    z, u = both[:, :cols], both[:, cols:]
    h, saved = B.dq_gate(z, u, save=True)
    dz, du = B.dq_gate_grad(h, saved)
    some = torch.tensor([0, 1, rows // 2, rows - 1], device=dev)
    a, ta = P.activation(z[some], "silu")[0], P.activation_bounds(z[some], "silu")[0]
    want, step = a * u[some].double(), P.half_step(torch.bfloat16)
    tol = ta * u[some].double().abs() + P.U * want.abs()
    assert bool(((h[some].double() - want).abs() <= tol + step * (want.abs() + tol) + 1e-37).all())
    a, ta = P.activation(P.held(z[some]), "silu")[0], P.activation_bounds(P.held(z[some]), "silu")[0]
    g = h[some].double()
    tol = ta * g.abs() + 4 * P.U * (g * a).abs()
    assert bool(((du[some].double() - g * a).abs() <= tol + step * ((g * a).abs() + tol) + 1e-37).all())


@pytest.mark.parametrize("rows,cols", [(1100000, 2048), (130001, 17000)])
def test_layer_norm_past_2_to_the_31_entries(dev, rows, cols):
    x = fill(rows, cols, dev, 3)
    assert x.numel() > 2 ** 31
    weight, bias = torch.linspace(0.5, 1.5, cols, device=dev), torch.linspace(-1, 1, cols, device=dev)
    y, saved = B.dq_layer_norm(x, weight, bias, save=True)
    some = torch.tensor([0, rows // 2, rows - 3, rows - 1], device=dev)
    bound = P.layer_norm_bound(x[some], weight, bias, 1e-5, torch.bfloat16)[0]
    assert bool(((y[some].double() - P.layer_norm(x[some], weight, bias, 1e-5)[0]).abs() <= bound).all())
    del y
    dy = torch.zeros_like(x)                       # all but a few rows count nothing in the sums over rows
    dy[some] = x[some].flip(1)
    got = B.dq_layer_norm_grad(dy, saved, weight)
    xv = P.held(x[some])
    wants = P.layer_norm_grad(dy[some], xv, saved.mean[some], saved.rstd[some], weight)
    bounds = P.layer_norm_grad_bounds(dy[some], xv, saved.mean[some], saved.rstd[some], weight, torch.bfloat16, torch.float32)
    assert bool(((got[0][some].double() - wants[0]).abs() <= bounds[0]).all())
    # a thread adds its rows of zeros to what it has: exact; the parts of 256 blocks are then at most 256 additions more
    for k in (1, 2):
        assert bool(((got[k].double() - wants[k]).abs() <= bounds[k] * (1 + 256 / 4)).all())


def test_weight_grad_of_many_tokens(dev):
    """dy past 2^31 entries; whole numbers in a few rows, so that sums are exact."""
    rows, outs, cols = 530001, 4100, 64
    g = torch.Generator(device=dev)
    g.manual_seed(4)
    x = torch.randint(-7, 8, (rows, cols), generator=g, device=dev).to(torch.bfloat16)
    dy = torch.zeros(rows, outs, dtype=torch.bfloat16, device=dev)
    assert dy.numel() > 2 ** 31
    some = torch.cat([torch.arange(0, 5, device=dev), torch.arange(rows // 2, rows // 2 + 70, device=dev), torch.arange(rows - 33, rows, device=dev)])
    dy[some] = torch.randint(-9, 10, (len(some), outs), generator=g, device=dev).to(torch.bfloat16)
    dw, db = B.dq_ckpt_weight_grad(dy, B.dq_ckpt_save(x), out=torch.empty(outs, cols, device=dev), bias=True)
    want, want_b = P.weight_grad(dy[some], P.held(x[some]))
    assert torch.equal(dw.double(), want) and torch.equal(db.double(), want_b)


def test_weight_grad_of_more_tiles_than_blocks(dev):
    """dw past 2^32 entries: more tiles than a grid has blocks, so that blocks take several."""
    rows, outs, cols = 3, 66001, 66304
    assert outs * cols > 2 ** 32 and -(-outs // 256) * -(-cols // 256) > 65536
    g = torch.Generator(device=dev)
    g.manual_seed(5)
    x = torch.randint(-7, 8, (rows, cols), generator=g, device=dev).to(torch.bfloat16)
    dy = torch.randint(-9, 10, (rows, outs), generator=g, device=dev).to(torch.bfloat16)
    ck = B.dq_ckpt_save(x)
    xv = B.dq_ckpt_load(ck)
    dw, db = B.dq_ckpt_weight_grad(dy, ck, bias=True)                    # bf16: of whole numbers up to 256 each is exact
    assert torch.equal(db.float(), dy.float().sum(0))
    for first in range(0, outs, 8192):
        part = dy[:, first:first + 8192].float()
        want = sum(part[t][:, None] * xv[t][None, :] for t in range(rows))
        assert torch.equal(dw[first:first + 8192].float(), want), first


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols,ld", [(8192, 8192), (8187, 8192), (8187, 8187), (8161, 8200)])
def test_large_calls_give_what_calls_over_parts_give(dev, dtype, cols, ld):
    rows, part = 9001, 643                         # the whole: 140 MiB and more a matrix; a part: 22 MiB at most
    both = fill(rows, 2 * ld, dev, 4).to(dtype)
    z, u = both[:, :cols], both[:, ld:ld + cols]
    own = [torch.full((rows, ld), 7.0, dtype=dtype, device=dev) for _ in range(4)]
    h, dz, du, back = [t[:, :cols] for t in own]
    ck = B.dq_ckpt_save(z)
    B.dq_ckpt_load(ck, dtype, out=back)
    _, saved = B.dq_gate(z, u, "gelu", save=True, out=h)
    B.dq_gate_grad(h, saved, dz, du)
    assert torch.equal(saved.z.data, ck.data)
    if ld > cols:
        assert all(bool((t[:, cols:] == 7.0).all()) for t in own)
    for k in range(0, rows, part):
        a = slice(k, min(rows, k + part))
        assert torch.equal(B.dq_ckpt_load(B.dq_ckpt_save(z[a]), dtype), back[a])
        want, kept = B.dq_gate(z[a], u[a], "gelu", save=True)
        wz, wu = B.dq_gate_grad(want, kept)
        assert torch.equal(want, h[a]) and torch.equal(wz, dz[a]) and torch.equal(wu, du[a])
        assert torch.equal(B.dq_gate(z[a], None, "silu"), B.dq_gate(z, None, "silu")[a]) if k == 0 else True


@pytest.mark.parametrize("dtype,weights", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("cols,ld", [(128, 128), (97, 128), (250, 256), (500, 504), (1000, 1000), (1029, 1032), (2048, 2048), (3000, 3000), (4096, 4096),
                                     (5000, 5008), (6151, 6152), (9001, 9008), (12300, 12304), (16384, 16384)])
def test_large_layer_norms(dev, dtype, weights, cols, ld):
    """x of 128 MiB and more, in every way that rows are kept."""
    rows = (1 << 27) // (cols * dtype.itemsize) + 5
    whole = fill(rows, ld, dev, 5).to(dtype)
    x = whole[:, :cols]
    weight, bias = torch.linspace(0.5, 1.5, cols, device=dev).to(weights), torch.linspace(-1, 1, cols, device=dev).to(weights)
    out = torch.full((rows, ld), 7.0, dtype=dtype, device=dev)
    y, saved = B.dq_layer_norm(x, weight, bias, save=True, out=out[:, :cols])
    some = torch.cat([torch.arange(0, rows, rows // 37, device=dev), torch.arange(rows - 3, rows, device=dev)]).unique()
    want, mean, rstd = P.layer_norm(x[some], weight, bias, 1e-5)
    bound, dk, dm = P.layer_norm_bound(x[some], weight, bias, 1e-5, dtype)
    assert bool(((y[some].double() - want).abs() <= bound).all())
    assert bool(((saved.mean[some].double() - mean.reshape(-1)).abs() <= dm.reshape(-1)).all())
    assert bool(((saved.rstd[some].double() - rstd.reshape(-1)).abs() <= (rstd * dk).reshape(-1)).all())
    assert torch.equal(saved.x.data, B.dq_ckpt_save(x).data)
    del y
    dy = torch.zeros_like(whole)[:, :cols]         # all but a few rows count nothing in the sums over rows
    dy[some] = x[some].flip(1)
    dx, dw, db = B.dq_layer_norm_grad(dy, saved, weight, out=out[:, :cols])
    xv = P.held(x[some])
    wants = P.layer_norm_grad(dy[some], xv, saved.mean[some], saved.rstd[some], weight)
    bounds = P.layer_norm_grad_bounds(dy[some], xv, saved.mean[some], saved.rstd[some], weight, dtype, weights)
    assert bool(((dx[some].double() - wants[0]).abs() <= bounds[0]).all())
    rest = torch.ones(rows, dtype=torch.bool, device=dev)
    rest[some] = False
    assert bool((dx[rest] == 0).all()) and (ld == cols or bool((out[:, cols:] == 7.0).all()))
    # a thread adds its rows of zeros to what it has: exact; the parts of 256 blocks are then at most 256 additions more
    for got, v, tol in ((dw, wants[1], bounds[1]), (db, wants[2], bounds[2])):
        assert bool(((got.double() - v).abs() <= tol * (1 + 256 / 4)).all())
