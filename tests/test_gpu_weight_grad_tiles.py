"""Weight gradients by tile: sizes that the library gives each of its tiles, unsplit, split over tokens and split many times, with ragged ends in
all three directions; which tile and how many splits each size gets is read off the launches here, so that another rule shows."""
import json
import os
import subprocess
import sys
import textwrap

import pytest
import torch

from paper_2602_08923_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# tokens, outs, columns: (a tile's edge, splits of the tokens) for fp32 and for bf16
CUTS = {
    (1029, 300, 515): ((64, 5), (64, 4)),
    (65537, 200, 136): ((64, 42), (64, 41)),
    (70, 4099, 4099): ((128, 1), (128, 1)),
    (300, 4099, 4099): ((128, 1), (128, 1)),
    (4111, 1101, 1499): ((128, 2), (128, 2)),
    (40000, 523, 1030): ((128, 11), (128, 11)),
    (70001, 260, 390): ((128, 21), (128, 21)),
    (1037, 3995, 4090): ((256, 1), (256, 1)),
    (8229, 1501, 2029): ((256, 5), (256, 5)),
    (60001, 390, 500): ((256, 63), (128, 16)),
}
SIZES = sorted(CUTS)


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield torch.device("cuda:0")
    torch.cuda.empty_cache()


def test_which_tile_each_size_gets(tmp_path):
    """From what a call would launch (tests/launch_recorder.c): blocks of 512 threads for the largest tile, one block to a tile and split."""
    so = str(tmp_path / "launch_recorder.so")
    subprocess.check_call(["gcc", "-O1", "-Wall", "-shared", "-fPIC", os.path.join(HERE, "launch_recorder.c"), "-o", so])
    body = f"""
        import ctypes as C, json, sys
        sys.path.insert(0, {os.path.dirname(HERE)!r})
        R = C.CDLL({so!r}, mode=C.RTLD_GLOBAL)
        from paper_2602_08923_amd import binding as B
        L = C.CDLL(B.LIB_PATH)
        class Launch(C.Structure):
            _fields_ = [("grid", C.c_uint32 * 3), ("block", C.c_uint32 * 3), ("args", C.c_uint64 * 8)]
        P, U, I, M = C.c_void_p, C.c_uint64, C.c_int, C.POINTER(B.Matrix)
        L.dq_ckpt_weight_grad_scratch_bytes.argtypes, L.dq_ckpt_weight_grad_scratch_bytes.restype = [I, U, U, U], C.c_size_t
        L.dq_ckpt_weight_grad.argtypes = [M, P, U, U, U, M, P, I, P, C.c_size_t, P]
        out = []
        for rows, outs, cols in {SIZES!r}:
            for t in (0, 1):
                need = L.dq_ckpt_weight_grad_scratch_bytes(t, rows, outs, cols)
                g, w = B.Matrix(1 << 50, t, outs), B.Matrix(3 << 50, t, cols)
                assert L.dq_ckpt_weight_grad(g, 2 << 50, rows, outs, cols, w, 4 << 50, 0, 5 << 50, need, None) == 0
                a = (Launch * 8)()
                n = R.recorded(a, 8)
                out.append((need, n, a[0].grid[0], a[0].block[0]))
        print(json.dumps(out))
    """
    got = subprocess.run([sys.executable, "-c", textwrap.dedent(body)], capture_output=True, text=True, timeout=300)
    assert got.returncode == 0, got.stderr
    want = []
    for rows, outs, cols in SIZES:
        for edge, splits in CUTS[rows, outs, cols]:
            tiles = -(-outs // edge) * -(-cols // edge)
            want.append([splits * (tiles * edge * edge + outs) * 4 if splits > 1 else 0, 2 if splits > 1 else 1, tiles * splits, 512 if edge == 256 else 256])
    assert json.loads(got.stdout) == want


def inside(rows, cols, dtype, dev):
    """A matrix inside a wider one, off 16-byte borders; the wider one holds 7 beside it."""
    whole = torch.full((rows, cols + 5), 7.0, dtype=dtype, device=dev)
    return whole, whole[:, 3:3 + cols]


def beside(whole, cols):
    return bool((whole[:, :3] == 7).all()) and bool((whole[:, 3 + cols:] == 7).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,outs,cols", SIZES)
def test_whole_numbers(dev, rows, outs, cols, dtype, out):
    """Small whole numbers: exact sums, rounded once to the output's type; with a bias, by itself and added to what is there."""
    g = torch.Generator(device=dev).manual_seed(rows + outs + cols)
    x = torch.randint(-7, 8, (rows, cols), generator=g, device=dev).to(torch.bfloat16)
    d = torch.randint(-9, 10, (rows, outs), generator=g, device=dev)
    assert 63 * rows + 200 < 2 ** 24
    dy = inside(rows, outs, TYPES[dtype], dev)[1]
    dy.copy_(d)
    ck = B.dq_ckpt_save(x)
    want = (d.double().t().contiguous() @ x.double()).float()
    want_b = d.double().sum(0).float()
    whole, dw = inside(outs, cols, TYPES[out], dev)
    db = torch.full((outs,), 7.0, dtype=TYPES[out], device=dev)
    B.dq_ckpt_weight_grad(dy, ck, out=dw, bias_out=db)
    assert bool((dw == want.to(dw.dtype)).all()) and bool((db == want_b.to(db.dtype)).all()) and beside(whole, cols)
    old = torch.randint(-100, 101, (outs, cols), generator=g, device=dev).float()
    dw.copy_(old)
    db.copy_(old[:, 0])
    B.dq_ckpt_weight_grad(dy, ck, out=dw, bias_out=db, accumulate=True)
    assert bool((dw == (want + old).to(dw.dtype)).all()) and bool((db == (want_b + old[:, 0]).to(db.dtype)).all()) and beside(whole, cols)
    dw.fill_(3.0)
    B.dq_ckpt_weight_grad(dy, ck, out=dw)
    assert bool((dw == want.to(dw.dtype)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,outs,cols", SIZES)
def test_every_digit_of_one_token(dev, rows, outs, cols):
    """fp32, one token to an output, the first and the last 64 tokens and others in between: 24 digits, all of the three parts that they are cut
    into, times powers of two come out as they are."""
    g = torch.Generator(device=dev).manual_seed(rows)
    x = torch.exp2(torch.randint(-3, 4, (rows, cols), generator=g, device=dev).float()) * (torch.randint(0, 2, (rows, cols), generator=g, device=dev) * 2 - 1)
    ck = B.dq_ckpt_save(x.to(torch.bfloat16))
    token = torch.randint(0, rows, (outs,), generator=g, device=dev)
    ends = torch.arange(min(64, rows), device=dev)
    places = torch.randperm(outs, generator=g, device=dev)[:2 * len(ends)]
    token[places] = torch.cat([ends, rows - 1 - ends])
    digits = torch.randint(2 ** 23, 2 ** 24, (outs,), generator=g, device=dev) | 1
    value = digits.float() * torch.exp2(torch.randint(-40, 10, (outs,), generator=g, device=dev).float())
    dy = torch.zeros(rows, outs, device=dev)
    dy[token, torch.arange(outs, device=dev)] = value
    dw, db = B.dq_ckpt_weight_grad(dy, ck, bias=True)
    assert bool((dw == value[:, None] * x[token]).all()) and torch.equal(db, value)
