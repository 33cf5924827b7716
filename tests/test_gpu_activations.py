"""8-bit activation checkpoints, weight gradients, layer norm and gates on the GPU against their formulas in 64 bits
(tests/plain_activations.py): codes, scales and loaded values exactly, computed numbers within bounds that count roundings."""
import pytest
import torch

from oracle import dq_oracle as O
from paper_2602_08923_amd import binding as B
from paper_2602_08923_amd import workloads
from tests import plain_activations as P

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U8 = torch.uint8


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def gen(dev, seed):
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return g


def acts(dev, rows, cols, dtype, seed, spread=1.0):
    g = gen(dev, seed)
    x = torch.randn(rows, cols, generator=g, device=dev) * torch.exp(spread * torch.randn(rows, 1, generator=g, device=dev))
    return (x * torch.where(torch.rand(1, cols, generator=g, device=dev) < 0.05, 20.0, 1.0)).to(dtype)


def part_of(x, before, after):
    """x as a part of a wider tensor whose other columns hold 7."""
    rows, cols = x.shape
    wide = torch.full((rows, before + cols + after), 7.0, dtype=x.dtype, device=x.device)
    wide[:, before:before + cols] = x
    return wide, wide[:, before:before + cols]


def within(got, want, bound, what):
    off = (got.double() - want).abs()
    worst = (off - bound).argmax()
    assert bool((off <= bound).all()), f"{what}: {got.reshape(-1)[worst]} for {want.reshape(-1)[worst]}, allowed {bound.reshape(-1)[worst]}"


def fields(ck):
    pitch = (ck.cols + 31) // 32 * 32
    codes = ck.data[:ck.rows * pitch].reshape(ck.rows, pitch).cpu()
    return codes, ck.data[ck.rows * pitch:B.dq_ckpt_bytes(ck.rows, ck.cols)].reshape(ck.rows, -1).cpu()


# ------------------------------------------------------------------------------------ checkpoints
SHAPES = [(1, 1), (1, 2048), (3, 31), (5, 32), (7, 33), (2, 40), (257, 255), (64, 515), (31, 2051), (1030, 8), (9, 8200)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_checkpoint_bytes_and_values(dev, rows, cols, dtype):
    x = acts(dev, rows, cols, TYPES[dtype], rows * 10007 + cols, spread=3.0)
    codes, scales, values = P.ckpt_fields(x)
    for y in (x, part_of(x, 1, 2)[1], part_of(x, 8, 0)[1]):
        ck = B.dq_ckpt_save(y)
        assert (ck.rows, ck.cols, ck.data.numel()) == (rows, cols, B.dq_ckpt_bytes(rows, cols))
        got = fields(ck)
        assert torch.equal(got[0], codes) and torch.equal(got[1], scales)
    for t in TYPES.values():                                             # exact in both types
        assert torch.equal(B.dq_ckpt_load(ck, t).double(), values)
        wide, out = part_of(torch.zeros(rows, cols, dtype=t, device=dev), 3, 5)
        assert B.dq_ckpt_load(ck, out=out) is out
        assert torch.equal(out.double(), values)
        assert bool((wide[:, :3] == 7).all()) and bool((wide[:, 3 + cols:] == 7).all())


def test_every_code_and_every_tie(dev):
    """Every E4M3 value, every middle between two of them and a step to either side, at the scales' ends and in between."""
    table = torch.tensor([m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** p for p in range(-6, 9) for m in range(8)][:119])
    mid = (table[1:] + table[:-1]) / 2
    v = torch.cat([table, mid, torch.nextafter(mid, torch.tensor(0.0)), torch.nextafter(mid, torch.tensor(1e9)), torch.tensor([449.0, 463.9, 464.0, 480.0, 511.9])])
    v = torch.cat([v, -v])
    v = torch.nn.functional.pad(v, (0, -len(v) % 31))
    rows = torch.cat([torch.full((len(v) // 31, 1), 256.0), v.reshape(-1, 31)], 1).reshape(-1, 32)
    for k in (-117, -60, 0, 3, 60, 118, 119):
        x = (rows.double() * 2.0 ** k).float()
        x = x[torch.isfinite(x).all(1)].to(dev)
        codes, scales, values = P.ckpt_fields(x)
        ck = B.dq_ckpt_save(x)
        got = fields(ck)
        assert torch.equal(got[0], codes) and torch.equal(got[1], scales) and torch.equal(B.dq_ckpt_load(ck).double(), values)


def test_tiny_huge_and_zero_blocks(dev):
    tiny = torch.tensor([2.0 ** -149, 2.0 ** -126, 2.0 ** -127, 2.0 ** -118, 2.0 ** -109, 2.0 ** -110 * 1.9, 0.0, -0.0] * 4, device=dev)
    huge = torch.full((32,), torch.finfo(torch.float32).max, device=dev)
    x = torch.stack([tiny, torch.zeros_like(tiny), huge, -huge, tiny.clamp(max=2.0 ** -126), torch.linspace(-1, 1, 32, device=dev) * 2.0 ** -108])
    codes, scales, values = P.ckpt_fields(x)
    ck = B.dq_ckpt_save(x)
    got = fields(ck)
    assert torch.equal(got[0], codes) and torch.equal(got[1], scales)
    assert int(got[1].min()) == 10 and int(got[1].max()) == 246
    loaded = B.dq_ckpt_load(ck)
    assert torch.equal(loaded.double(), values) and torch.equal(B.dq_ckpt_load(ck, torch.bfloat16).double(), values)
    assert bool(((loaded == 0) | (loaded.abs() >= 2.0 ** -126)).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_and_nan_stay_in_their_block(dev, dtype):
    x = acts(dev, 4, 100, TYPES[dtype], 5)
    want = P.ckpt_fields(x)[2]
    x[0, 3], x[1, 40], x[2, 99], x[3, 64] = float("inf"), float("nan"), float("-inf"), float("nan")
    codes, scales, values = P.ckpt_fields(x)
    ck = B.dq_ckpt_save(x)
    got = fields(ck)
    assert torch.equal(got[0], codes) and torch.equal(got[1], scales)
    for t in TYPES.values():
        loaded = B.dq_ckpt_load(ck, t).double()
        assert torch.equal(torch.isnan(loaded), torch.isnan(values)) and torch.equal(loaded[~torch.isnan(loaded)], want[~torch.isnan(loaded)])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_checkpoint_is_the_mx_codecs_bytes(dev, dtype):
    x = workloads.draw(workloads.CONFIGS[2], 0, device="cpu", entries=256 * 77).float().to(TYPES[dtype]).to(dev)
    packed = B.dq_mx_compress(B.DQ_MXFP8_E4M3, x)
    ck = B.dq_ckpt_save(x.reshape(77, 256))
    assert torch.equal(ck.data, packed[:ck.data.numel()])
    assert torch.equal(B.dq_ckpt_load(ck).reshape(-1), B.dq_mx_decompress(B.DQ_MXFP8_E4M3, packed, x.numel()))
    assert O.mx_packed_bytes(1, x.numel()) >= ck.data.numel()


# ------------------------------------------------------------------------------------ weight gradient
WGRAD = [(1, 1, 1), (1, 64, 64), (2, 300, 33), (5, 515, 2048), (31, 65, 127), (33, 64, 64), (64, 129, 257), (100, 8, 700), (257, 130, 96),
         (1000, 256, 256), (1029, 300, 515), (4097, 72, 40), (9000, 7, 9)]


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,outs,cols", WGRAD)
def test_weight_grad(dev, rows, outs, cols, dtype, out):
    x = acts(dev, rows, cols, torch.bfloat16, rows + outs + cols)
    dy = acts(dev, rows, outs, TYPES[dtype], rows + outs + cols + 1) * 1e-3
    ck = B.dq_ckpt_save(x)
    xv = P.held(x)
    dw = torch.empty(outs, cols, dtype=TYPES[out], device=dev)
    got = B.dq_ckpt_weight_grad(dy, ck, out=dw, bias=True)
    assert got[0] is dw and got[1].dtype == dw.dtype
    (want, want_b), (tol, tol_b) = P.weight_grad(dy, xv), P.weight_grad_bounds(dy, xv, TYPES[out])
    within(got[0], want, tol, "dw")
    within(got[1], want_b, tol_b, "db")
    again = B.dq_ckpt_weight_grad(dy, ck, out=torch.empty_like(dw), bias=True)      # the same bits each time
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    if dtype == out:
        alone = B.dq_ckpt_weight_grad(dy, ck)
        assert alone.dtype == dy.dtype and torch.equal(alone, got[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,outs,cols", [(1, 5, 3), (37, 100, 97), (640, 257, 300), (2500, 64, 130), (70, 1100, 700), (1500, 600, 520)])
def test_weight_grad_of_whole_numbers_is_exact(dev, rows, outs, cols, dtype):
    """Small whole numbers: every product and sum is one of binary32, whatever the order."""
    g = gen(dev, rows)
    x = torch.randint(-15, 16, (rows, cols), generator=g, device=dev).to(torch.bfloat16)
    dy = torch.randint(-40, 41, (rows, outs), generator=g, device=dev).to(TYPES[dtype])
    if dtype == "f32":
        dy += torch.randint(0, 2, (rows, outs), generator=g, device=dev) * 2.0 ** -8        # more digits than a bf16 number has
    xs, ds = part_of(x, 3, 6)[1], part_of(dy, 5, 2)[1]
    ck = B.dq_ckpt_save(xs)
    xv = P.held(x)                               # whole numbers too: where 15 is a block's largest, 15 * 2^(8 - 3) = 480 saturates at 448, 14
    assert torch.equal(B.dq_ckpt_load(ck).double(), xv)
    want, want_b = P.weight_grad(dy, xv)
    wide, out = part_of(torch.empty(outs, cols, device=dev), 2, 3)
    for d in (dy, ds):
        out.zero_()
        dw, db = B.dq_ckpt_weight_grad(d, ck, out=out, bias=True)
        assert torch.equal(dw.double(), want) and torch.equal(db.double(), want_b)
        assert bool((wide[:, :2] == 7).all()) and bool((wide[:, 2 + cols:] == 7).all())
    db = torch.full((outs,), 3.0, device=dev)
    B.dq_ckpt_weight_grad(dy, ck, out=out, bias_out=db, accumulate=True)
    assert torch.equal(out.double(), 2 * want) and torch.equal(db.double(), want_b + 3)


def test_weight_grad_of_no_rows_and_of_several_dimensions(dev):
    ck = B.dq_ckpt_save(torch.empty(0, 40, device=dev))
    dw, db = B.dq_ckpt_weight_grad(torch.empty(0, 9, device=dev), ck, bias=True)
    assert dw.shape == (9, 40) and not dw.any() and not db.any()
    out = torch.ones(9, 40, device=dev)
    B.dq_ckpt_weight_grad(torch.empty(0, 9, device=dev), ck, out=out, accumulate=True)
    assert bool((out == 1).all())
    x, dy = acts(dev, 60, 70, torch.bfloat16, 1), acts(dev, 60, 50, torch.bfloat16, 2)
    want = B.dq_ckpt_weight_grad(dy, B.dq_ckpt_save(x))
    assert torch.equal(B.dq_ckpt_weight_grad(dy.reshape(3, 20, 50), B.dq_ckpt_save(x.reshape(4, 15, 70))), want)


def test_weight_grad_keeps_bad_tokens_to_their_rows_and_columns(dev):
    """NaN in one output's gradient and in one block of the inputs: the other rows and columns are as without."""
    x, dy = acts(dev, 300, 256, torch.bfloat16, 3), acts(dev, 300, 200, torch.bfloat16, 4)
    clean = B.dq_ckpt_weight_grad(dy, B.dq_ckpt_save(x))
    x[17, 70], dy[250, 9] = float("inf"), float("nan")
    got = B.dq_ckpt_weight_grad(dy, B.dq_ckpt_save(x))
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[9], bad[:, 64:96] = True, True
    assert torch.equal(torch.isnan(got), bad) and torch.equal(got[~bad], clean[~bad])


# ------------------------------------------------------------------------------------ layer norm
NORM = [(1, 1), (1, 2048), (3, 31), (5, 8), (2, 40), (257, 515), (700, 768), (33, 1031), (1030, 64), (64, 4096), (19, 6151), (3, 9000), (2, 33000), (2100, 257)]


@pytest.mark.parametrize("dtype,weights", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,cols", NORM)
def test_layer_norm(dev, rows, cols, dtype, weights):
    t, w = TYPES[dtype], TYPES[weights]
    x, dy = acts(dev, rows, cols, t, rows + cols) + 0.5, acts(dev, rows, cols, t, rows + cols + 1)
    weight, bias = (acts(dev, 1, cols, w, 3) * 0.2 + 1).reshape(-1), acts(dev, 1, cols, w, 4).reshape(-1)
    bound, dk, dm = P.layer_norm_bound(x, weight, bias, 1e-5, t)
    want, mean, rstd = P.layer_norm(x, weight, bias, 1e-5)
    y = B.dq_layer_norm(x, weight, bias)
    within(y, want, bound, "y")
    wide, part = part_of(x, 3, 1)
    again, saved = B.dq_layer_norm(part, weight, bias, 1e-5, save=True)
    assert torch.equal(again, y)
    within(saved.mean, mean.reshape(-1), dm.reshape(-1), "mean")
    within(saved.rstd, rstd.reshape(-1), (rstd * dk).reshape(-1), "rstd")
    ck = B.dq_ckpt_save(x)
    assert torch.equal(saved.x.data, ck.data) and saved.x[1:] == ck[1:]
    xv = P.held(x)
    for wt in (weight, None):
        dx, dw, db = B.dq_layer_norm_grad(dy, saved, wt)
        wants = P.layer_norm_grad(dy, xv, saved.mean, saved.rstd, wt)
        bounds = P.layer_norm_grad_bounds(dy, xv, saved.mean, saved.rstd, wt, t, w)
        within(dx, wants[0], bounds[0], "dx")
        if wt is None:
            assert dw is None and db is None
        else:
            assert dw.dtype == w and db.dtype == w
            within(dw, wants[1], bounds[1], "dweight")
            within(db, wants[2], bounds[2], "dbias")
            keep = dx, dw, db
    _, dpart = part_of(dy, 1, 4)
    wout, out = part_of(torch.empty_like(dx), 5, 2)
    wo, bo = torch.full((cols,), 2.0, device=dev, dtype=w), torch.full((cols,), -1.0, device=dev, dtype=w)
    got = B.dq_layer_norm_grad(dpart, saved, weight, out=out, weight_out=wo, bias_out=bo, accumulate=True)
    assert got[0] is out and torch.equal(out, keep[0])
    assert bool((wout[:, :5] == 7).all()) and bool((wout[:, 5 + cols:] == 7).all())
    within(wo, wants_plus(dy, xv, saved, weight, 1, 2.0), bounds_plus(dy, xv, saved, weight, t, w, 1, 2.0), "dweight added")
    within(bo, wants_plus(dy, xv, saved, weight, 2, -1.0), bounds_plus(dy, xv, saved, weight, t, w, 2, -1.0), "dbias added")


def wants_plus(dy, xv, saved, weight, k, start):
    return P.layer_norm_grad(dy, xv, saved.mean, saved.rstd, weight)[k] + start


def bounds_plus(dy, xv, saved, weight, t, w, k, start):
    """The sum in binary32 (bound taken there), one addition more, one rounding."""
    want = P.layer_norm_grad(dy, xv, saved.mean, saved.rstd, weight)[k] + start
    off = P.layer_norm_grad_bounds(dy, xv, saved.mean, saved.rstd, weight, t, torch.float32)[k] + P.U * want.abs()
    return off + P.half_step(w) * (want.abs() + off)


def test_layer_norm_without_weights_and_of_several_dimensions(dev):
    x = acts(dev, 24, 100, torch.float32, 9)
    plain = B.dq_layer_norm(x)
    within(plain, P.layer_norm(x, None, None, 1e-5)[0], P.layer_norm_bound(x, None, None, 1e-5, torch.float32)[0], "y")
    bias = acts(dev, 1, 100, torch.bfloat16, 2).reshape(-1)
    within(B.dq_layer_norm(x, bias=bias), P.layer_norm(x, None, bias, 1e-5)[0], P.layer_norm_bound(x, None, bias, 1e-5, torch.float32)[0], "y")
    y, saved = B.dq_layer_norm(x.reshape(2, 3, 4, 100), save=True)
    assert y.shape == (2, 3, 4, 100) and torch.equal(y.reshape(24, 100), plain)
    dx, _, _ = B.dq_layer_norm_grad(x.reshape(4, 6, 100), saved)
    assert dx.shape == (4, 6, 100)
    none = B.dq_layer_norm(torch.empty(0, 100, device=dev), save=True)
    dx, dw, db = B.dq_layer_norm_grad(torch.empty(0, 100, device=dev), none[1], bias)
    assert dx.shape == (0, 100) and not dw.any() and not db.any()


@pytest.mark.parametrize("cols", [64, 515, 4096, 9000])
def test_layer_norm_of_constant_far_and_bad_rows(dev, cols):
    """A row of one value (rstd is 1 / sqrt(eps)), a row far from zero, and rows with an infinity and a NaN, which stay theirs."""
    x = acts(dev, 6, cols, torch.float32, 11)
    x[0], x[1] = 3.0, 10000.0 + torch.rand(cols, device=dev, generator=gen(dev, 1))
    clean, saved = B.dq_layer_norm(x, save=True)
    within(clean, P.layer_norm(x, None, None, 1e-5)[0], P.layer_norm_bound(x, None, None, 1e-5, torch.float32)[0], "y")
    within(saved.rstd[:1], torch.full((1,), 1e-5, device=dev, dtype=torch.float64).rsqrt(), torch.tensor([1e-4], device=dev), "rstd")
    x[2, 5], x[4, cols - 1] = float("inf"), float("nan")
    y, bad = B.dq_layer_norm(x, save=True)
    keep = torch.tensor([0, 1, 3, 5], device=dev)
    assert torch.equal(y[keep], clean[keep]) and torch.equal(bad.mean[keep], saved.mean[keep])
    assert bool(torch.isnan(y[4]).all()) and not bool(torch.isfinite(bad.mean[2])) and not bool(torch.isfinite(y[2]).any())
    dy = acts(dev, 6, cols, torch.float32, 12)
    a, b = B.dq_layer_norm_grad(dy, saved)[0], B.dq_layer_norm_grad(dy, bad)[0]
    assert torch.equal(a[keep], b[keep]) and bool(torch.isnan(b[2]).any()) and bool(torch.isnan(b[4]).all())


# ------------------------------------------------------------------------------------ gates
@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 2048), (3, 31), (33, 1000), (64, 515), (300, 256), (7, 8200)])
def test_gate(dev, rows, cols, dtype, kind):
    t = TYPES[dtype]
    both = acts(dev, rows, 2 * cols, t, rows + cols)
    z, u, dh = both[:, :cols], both[:, cols:], acts(dev, rows, cols, t, 5)
    step = P.half_step(t)
    a, _ = P.activation(z, kind)
    ta, _ = P.activation_bounds(z, kind)
    h, saved = B.dq_gate(z, kind=kind, save=True)
    assert saved.u is None and torch.equal(h, B.dq_gate(z.contiguous(), None, kind))
    within(h, a, ta + step * (a.abs() + ta), "h")
    hu, gated = B.dq_gate(z, u, kind, save=True)
    ud = u.double()
    want = a * ud
    tol = ta * ud.abs() + P.U * want.abs()
    within(hu, want, tol + step * (want.abs() + tol) + 1e-37, "h")
    assert torch.equal(hu, B.dq_gate(z, u, kind))
    for ck, x in ((saved.z, z), (gated.z, z), (gated.u, u)):
        assert torch.equal(ck.data, B.dq_ckpt_save(x).data)
    zv, uv, g = P.held(z), P.held(u), dh.double()
    a, d = P.activation(zv, kind)
    ta, td = P.activation_bounds(zv, kind)
    dz, none = B.dq_gate_grad(dh, saved)
    assert none is None
    within(dz, g * d, td * g.abs() + 3 * P.U * (g * d).abs() + step * (g * d).abs() * 1.01 + step * td * g.abs() + 1e-37, "dz")
    wide = torch.full((rows, 2 * cols), 7.0, dtype=t, device=dev)
    dz, du = B.dq_gate_grad(dh, gated, z_out=wide[:, :cols], u_out=wide[:, cols:])        # side by side, as z and u lie
    for got, want, tol in ((dz, g * uv * d, td * (g * uv).abs()), (du, g * a, ta * g.abs())):
        tol = tol + 4 * P.U * want.abs()
        within(got, want, tol + step * (want.abs() + tol) + 1e-37, "dz, du")


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gate_far_out(dev, kind):
    """Far from zero the activation is zero or its argument, and its derivative zero or one; nothing overflows on the way."""
    z = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 20.0, -20.0, 87.0, -87.0, 89.0, -89.0, 104.0, -104.0, 1e4, -1e4, 1e38, -1e38], device=dev)
    h, saved = B.dq_gate(z, kind=kind, save=True)
    want, tol = P.activation(z, kind)[0], P.activation_bounds(z, kind)[0]
    assert bool(torch.isfinite(h).all())
    within(h, want, tol.clamp(max=1e30) + 2 * P.U * want.abs() + 1e-37, "h")
    for v in (1e4, -1e4, 1e38, -1e38, 0.0):
        big = torch.full((32,), v, device=dev)
        dz, _ = B.dq_gate_grad(torch.ones_like(big), B.dq_gate(big, kind=kind, save=True)[1])
        assert bool((dz == (0.5 if v == 0 else float(v > 0))).all())


# ------------------------------------------------------------------------------------ together
def block(x, p, save=True):
    """A pre-norm gated feed-forward block: x + down(act(a) * b), (a, b) = up(norm(x))."""
    f = p["down"].shape[1]
    y, norm = B.dq_layer_norm(x, p["weight"], p["bias"], save=True)
    ck = B.dq_ckpt_save(y)
    ab = y @ p["up"].t()
    h, gate = B.dq_gate(ab[:, :f], ab[:, f:], "silu", save=True)
    return x + h @ p["down"].t(), (norm, ck, gate, B.dq_ckpt_save(h), ab, y, h)


def block_back(dout, p, saved):
    norm, ck, gate, ch = saved[:4]
    f = p["down"].shape[1]
    down = B.dq_ckpt_weight_grad(dout, ch)
    dab = torch.empty(dout.shape[0], 2 * f, dtype=dout.dtype, device=dout.device)
    dh = dout @ p["down"]
    B.dq_gate_grad(dh, gate, z_out=dab[:, :f], u_out=dab[:, f:])
    up = B.dq_ckpt_weight_grad(dab, ck)
    dy = dab @ p["up"]
    dx, dw, db = B.dq_layer_norm_grad(dy, norm, p["weight"])
    return {"x": dout + dx, "weight": dw, "bias": db, "up": up, "down": down}


def params(dev, d, f, dtype, seed=1):
    g = gen(dev, seed)
    return {"weight": (1 + 0.1 * torch.randn(d, generator=g, device=dev)).to(dtype), "bias": (0.1 * torch.randn(d, generator=g, device=dev)).to(dtype),
            "up": (torch.randn(2 * f, d, generator=g, device=dev) / d ** 0.5).to(dtype), "down": (torch.randn(d, f, generator=g, device=dev) / f ** 0.5).to(dtype)}


def test_a_block_of_them_together(dev):
    """Each step's output against 64 bits on the values that the step was given, and the whole against a backward pass that keeps
    activations whole: apart by what 8 bits lose (each entry by 2^-4 of itself at most, most by less), no more."""
    d, f, rows = 96, 160, 513
    p = params(dev, d, f, torch.float32)
    x, dout = acts(dev, rows, d, torch.float32, 3, 0.2), acts(dev, rows, d, torch.float32, 4, 0.2)
    out, saved = block(x, p)
    got = block_back(dout, p, saved)
    q = {k: v.double().requires_grad_() for k, v in p.items()}
    xd = x.double().requires_grad_()
    y = P.layer_norm(xd, q["weight"], q["bias"], 1e-5)[0]
    ab = y @ q["up"].t()
    whole = xd + (torch.sigmoid(ab[:, :f]) * ab[:, :f] * ab[:, f:]) @ q["down"].t()
    (whole * dout.double()).sum().backward()
    assert float((out.double() - whole.detach()).norm() / whole.detach().norm()) < 1e-5
    for name, want in [("x", xd.grad)] + [(k, v.grad) for k, v in q.items()]:
        off = float((got[name].double() - want).norm() / want.norm())
        assert off < 2.0 ** -4, (name, off)
    assert float((got["up"].double() - q["up"].grad).norm()) > 0                # 8 bits were used


def test_a_captured_block_replays(dev):
    """Forward and backward in one graph, on new inputs each time, the program's own work in between."""
    d, f, rows = 256, 320, 300
    p = params(dev, d, f, torch.bfloat16)
    x, dout = acts(dev, rows, d, torch.bfloat16, 3), acts(dev, rows, d, torch.bfloat16, 4)
    want = block_back(dout, p, block(x, p)[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block_back(dout, p, block(x, p)[1])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = block_back(dout, p, block(x, p)[1])
    for seed in (3, 20, 21, 22):
        x.copy_(acts(dev, rows, d, torch.bfloat16, seed))
        dout.copy_(acts(dev, rows, d, torch.bfloat16, seed + 1))
        graph.replay()
        torch.cuda.synchronize()
        held = {k: v.clone() for k, v in got.items()}
        want = block_back(dout, p, block(x, p)[1])
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(held[k], want[k]), (seed, k)


def test_on_another_stream(dev):
    x, dy = acts(dev, 2000, 300, torch.bfloat16, 3), acts(dev, 2000, 200, torch.bfloat16, 4)
    want = B.dq_ckpt_weight_grad(dy, B.dq_ckpt_save(x), bias=True)
    y, saved = B.dq_layer_norm(x, save=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = B.dq_ckpt_weight_grad(dy, B.dq_ckpt_save(x), bias=True)
        again, s2 = B.dq_layer_norm(x, save=True)
        back = B.dq_layer_norm_grad(x, s2, torch.ones(300, device=dev))
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(again, y)
    for a, b in zip(back, B.dq_layer_norm_grad(x, saved, torch.ones(300, device=dev))):
        assert torch.equal(a, b)


def test_gradients_against_differences(dev):
    """On activations that 8 bits hold, the gradients are those of the formulas: central differences in 64 bits of sum(dy * f(x)).
    A difference with a step s is off by s^2 / 6 of the third derivative (a few units here) and 2^-52 / s by rounding."""
    rows, cols, s = 6, 40, 1e-4
    x = P.held(acts(dev, rows, cols, torch.float32, 7, 0.1).clamp(-4, 4)).float()
    dy = acts(dev, rows, cols, torch.float32, 8, 0.1)
    weight, bias = (acts(dev, 1, cols, torch.float32, 3) * 0.1 + 1).reshape(-1), acts(dev, 1, cols, torch.float32, 4).reshape(-1)

    def difference(f, v):
        v = v.double()
        out = torch.empty_like(v)
        for k in range(v.numel()):
            e = torch.zeros_like(v).reshape(-1)
            e[k] = s
            out.view(-1)[k] = ((f(v + e.view_as(v)) - f(v - e.view_as(v))) * dy.double()).sum() / (2 * s)
        return out

    _, saved = B.dq_layer_norm(x, weight, bias, save=True)
    dx, dw, db = B.dq_layer_norm_grad(dy, saved, weight)
    for got, want in ((dx, difference(lambda v: P.layer_norm(v, weight, bias, 1e-5)[0], x)), (dw, difference(lambda v: P.layer_norm(x, v, bias, 1e-5)[0], weight)),
                      (db, difference(lambda v: P.layer_norm(x, weight, v, 1e-5)[0], bias))):
        assert float((got.double() - want).abs().max()) < 2e-5 * float(want.abs().max())
    for kind in ("silu", "gelu"):
        z, u = x, x.flip(0).contiguous()
        dz, du = B.dq_gate_grad(dy, B.dq_gate(z, u, kind, save=True)[1])
        for got, want in ((dz, difference(lambda v: P.activation(v, kind)[0] * u.double(), z)), (du, difference(lambda v: P.activation(z, kind)[0] * v, u))):
            assert float((got.double() - want).abs().max()) < 2e-5 * float(want.abs().max())
    w = acts(dev, 5, cols, torch.float32, 9)
    d5 = acts(dev, rows, 5, torch.float32, 10)
    dwl = B.dq_ckpt_weight_grad(d5, B.dq_ckpt_save(x))
    want = torch.empty(5, cols, dtype=torch.float64, device=dev)
    for k in range(w.numel()):
        e = torch.zeros_like(w, dtype=torch.float64).reshape(-1)
        e[k] = s
        want.view(-1)[k] = ((x.double() @ (2 * e.view_as(w)).t()) * d5.double()).sum() / (2 * s)
    assert float((dwl.double() - want).abs().max()) < 2e-5 * float(want.abs().max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 100), (33, 128), (5000, 129), (70, 256), (9, 200), (40000, 17), (20001, 250), (9000, 500), (4100, 1500), (5000, 2048), (4097, 1025), (2500, 3000), (600, 4099), (2200, 5000), (700, 12300), (600, 16384), (300, 8193)])
def test_layer_norm_of_every_way_to_keep_rows(dev, rows, cols, dtype):
    """Short rows that share a wave, and blocks that take several rows."""
    t = TYPES[dtype]
    x, dy = acts(dev, rows, cols, t, rows + cols) + 0.5, acts(dev, rows, cols, t, rows + cols + 1)
    weight, bias = (acts(dev, 1, cols, t, 3) * 0.2 + 1).reshape(-1), acts(dev, 1, cols, t, 4).reshape(-1)
    y, saved = B.dq_layer_norm(x, weight, bias, save=True)
    bound, dk, dm = P.layer_norm_bound(x, weight, bias, 1e-5, t)
    want, mean, rstd = P.layer_norm(x, weight, bias, 1e-5)
    within(y, want, bound, "y")
    within(saved.mean, mean.reshape(-1), dm.reshape(-1), "mean")
    within(saved.rstd, rstd.reshape(-1), (rstd * dk).reshape(-1), "rstd")
    assert torch.equal(saved.x.data, B.dq_ckpt_save(x).data)
    xv = P.held(x)
    got = B.dq_layer_norm_grad(dy, saved, weight)
    wants = P.layer_norm_grad(dy, xv, saved.mean, saved.rstd, weight)
    bounds = P.layer_norm_grad_bounds(dy, xv, saved.mean, saved.rstd, weight, t, t)
    for g, v, tol, what in zip(got, wants, bounds, ("dx", "dweight", "dbias")):
        within(g, v, tol, what)


def test_captured_gradients_add_up(dev):
    """Gradients added to a bucket inside a graph: each replay adds once more, split sums and joined parts among them; whole numbers, exact."""
    rows, outs, cols = 5000, 70, 90
    g = gen(dev, 1)
    x = torch.randint(-7, 8, (rows, cols), generator=g, device=dev).to(torch.bfloat16)
    dy = torch.randint(-9, 10, (rows, outs), generator=g, device=dev).to(torch.bfloat16)
    assert B.lib().dq_ckpt_weight_grad_scratch_bytes(B.DQ_BF16, rows, outs, cols) > 0
    want, want_b = P.weight_grad(dy, P.held(x))
    dw, db = torch.zeros(outs, cols, device=dev), torch.zeros(outs, device=dev)
    weight = torch.ones(cols, device=dev)
    bias_sum = torch.zeros(cols, device=dev)
    weight_sum = torch.zeros(cols, device=dev)

    def step():
        ck = B.dq_ckpt_save(x)
        B.dq_ckpt_weight_grad(dy, ck, out=dw, bias_out=db, accumulate=True)
        _, saved = B.dq_layer_norm(x, weight, save=True)
        B.dq_layer_norm_grad(x, saved, weight, weight_out=weight_sum, bias_out=bias_sum, accumulate=True)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    times = 1
    for _ in range(4):
        graph.replay()
        other = B.dq_ckpt_weight_grad(dy.flip(0).contiguous(), B.dq_ckpt_save(x), bias=True)     # the program's own work between replays
        torch.cuda.synchronize()
        times += 1
        assert torch.equal(dw.double(), times * want) and torch.equal(db.double(), times * want_b), times
        assert torch.equal(bias_sum.double(), times * x.double().sum(0)), times
        assert torch.equal(other[1].double(), want_b.to(torch.bfloat16).double())


def test_two_graphs_of_one_pool_and_two_streams_at_once(dev):
    x, dy = [acts(dev, 3000, 200, torch.bfloat16, s) for s in (1, 2)], [acts(dev, 3000, 100, torch.bfloat16, s) for s in (3, 4)]

    def work(k):
        y, saved = B.dq_layer_norm(x[k], save=True)
        return B.dq_ckpt_weight_grad(dy[k], B.dq_ckpt_save(y), bias=True) + (B.dq_layer_norm_grad(x[k], saved, torch.ones(200, device=dev))[1],)

    want = [[t.clone() for t in work(k)] for k in (0, 1)]
    torch.cuda.synchronize()
    graphs, got, pool = [], [], torch.cuda.graph_pool_handle()
    for k in (0, 1):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[k], pool=pool):
            got.append(work(k))
    for k in (0, 1, 1, 0, 1):                       # one after the other, as graphs that share a pool are replayed
        graphs[k].replay()
        torch.cuda.synchronize()
        for a, b in zip(got[k], want[k]):
            assert torch.equal(a, b)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        outs = []
        for k, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                outs.append(work(k))
        torch.cuda.synchronize()
        for k in (0, 1):
            for a, b in zip(outs[k], want[k]):
                assert torch.equal(a, b)


def test_out_arguments_and_refusals_of_shapes(dev):
    x = acts(dev, 6, 64, torch.bfloat16, 1)
    ck = B.dq_ckpt_save(x)
    out = torch.zeros(B.dq_ckpt_bytes(6, 64) + 32, dtype=torch.uint8, device=dev)
    again = B.dq_ckpt_save(x, out)
    assert again.data is out and torch.equal(out[:ck.data.numel()], ck.data) and not out[ck.data.numel():].any()
    _, saved = B.dq_layer_norm(x, save=True)
    h, gate = B.dq_gate(x, x.flip(0).contiguous(), save=True)
    w = torch.ones(64, device=dev)
    for call, match in [
        (lambda: B.dq_ckpt_save(x.t()), "side by side"),
        (lambda: B.dq_ckpt_save(x[:1].expand(6, 64)), "not overlap"),
        (lambda: B.dq_ckpt_save(x.reshape(2, 3, 64)[:, :2]), "one distance"),
        (lambda: B.dq_ckpt_save(x.half()), "float32 or bfloat16"),
        (lambda: B.dq_ckpt_save(x, out[:100]), "all its bytes"),
        (lambda: B.dq_ckpt_save(x, out[8:]), "aligned"),
        (lambda: B.dq_ckpt_save(x[0, 0]), "dimension"),
        (lambda: B.dq_ckpt_load(ck, torch.float16), "float32 or bfloat16"),
        (lambda: B.dq_ckpt_load(ck, out=torch.empty(6, 63, device=dev)), "another shape"),
        (lambda: B.dq_ckpt_load(B.Checkpoint(ck.data, 7, 64)), "all its bytes"),
        (lambda: B.dq_ckpt_load(B.Checkpoint(ck.data, -1, 64)), "not negative"),
        (lambda: B.dq_ckpt_weight_grad(x[:5], ck), "rows"),
        (lambda: B.dq_ckpt_weight_grad(x, ck, out=torch.empty(64, 63, device=dev)), "another shape"),
        (lambda: B.dq_ckpt_weight_grad(x, ck, accumulate=True), "give them"),
        (lambda: B.dq_ckpt_weight_grad(x, ck, out=torch.empty(64, 64, device=dev), bias=True, accumulate=True), "give them"),
        (lambda: B.dq_ckpt_weight_grad(x, ck, bias_out=torch.empty(63, dtype=x.dtype, device=dev)), "bias_out"),
        (lambda: B.dq_layer_norm(x, torch.ones(63, device=dev)), "weight"),
        (lambda: B.dq_layer_norm(x, w, w.bfloat16()), "bias"),
        (lambda: B.dq_layer_norm(x, eps=-1.0), "invalid"),
        (lambda: B.dq_layer_norm(x, out=x), "invalid"),
        (lambda: B.dq_layer_norm(x, out=torch.empty(6, 64, device=dev)), "another type"),
        (lambda: B.dq_layer_norm_grad(x[:5], saved, w), "another shape"),
        (lambda: B.dq_layer_norm_grad(x, saved, w, accumulate=True), "give them"),
        (lambda: B.dq_layer_norm_grad(x, saved, None, weight_out=w), "without a weight"),
        (lambda: B.dq_layer_norm_grad(x, saved, w, weight_out=w), "invalid"),
        (lambda: B.dq_gate(x, x[:, :32]), "another shape"),
        (lambda: B.dq_gate(x, x.float()), "another type"),
        (lambda: B.dq_gate_grad(x[:5], gate), "another shape"),
        (lambda: B.dq_gate_grad(x, gate._replace(u=None), u_out=torch.empty_like(x)), "no u"),
        (lambda: B.dq_gate_grad(x, gate, z_out=h, u_out=h), "invalid"),
        (lambda: B.dq_gate_grad(x, gate, z_out=x), "invalid"),
        (lambda: B.dq_layer_norm(x, w.cpu()), "different devices"),
    ]:
        with pytest.raises(B.DqError, match=match):
            call()
    torch.cuda.synchronize()
