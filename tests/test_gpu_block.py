"""The feed-forward block whose activations wait in 8-bit checkpoints (block.py): its gradients step by step against 64 bits, its
buckets, and the all-reduce of what its workers leave."""
import json
import subprocess
import sys
import os

import pytest
import torch

from paper_2602_08923_amd import allreduce as A
from paper_2602_08923_amd import binding as B
from paper_2602_08923_amd import block
from tests import plain_activations as P

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def within(got, want, bound, what):
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), (what, float((off - bound).max()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d,f,rows", [(96, 130, 200), (33, 17, 65), (256, 512, 1)])
def test_a_blocks_gradients(dev, d, f, rows, dtype):
    b = block.Block(d, f, dtype, seed=3, device=dev)
    x, target = block.tokens(d, rows, 0, dtype, device=dev)
    out, (norm, sy, gate, sh) = b.forward(x)
    dout = out - target
    bucket = torch.full((b.bucket_entries(4),), 5.0, dtype=dtype, device=dev)
    dx = b.backward(dout, (norm, sy, gate, sh), bucket)
    g = b.views(bucket)
    # the steps, each from what it was given
    p = b.params
    hv, yv, zv, uv = (B.dq_ckpt_load(c).double() for c in (sh, sy, gate.z, gate.u))
    within(g["down"], P.weight_grad(dout, hv)[0], P.weight_grad_bounds(dout, hv, dtype)[0], "down")
    dh = dout @ p["down"]
    dz, du = B.dq_gate_grad(dh, gate)
    (a, da), (ta, td) = P.activation(zv, "silu"), P.activation_bounds(zv, "silu")
    step, dhd = P.half_step(dtype), dh.double()
    for got, want, tol in ((dz, dhd * uv * da, td * (dhd * uv).abs()), (du, dhd * a, ta * dhd.abs())):
        tol = tol + 4 * P.U * want.abs()
        within(got, want, tol + step * (want.abs() + tol) + 1e-37, "gate")
    dab = torch.cat([dz, du], 1)
    within(g["up"], P.weight_grad(dab, yv)[0], P.weight_grad_bounds(dab, yv, dtype)[0], "up")
    dy, xv = dab @ p["up"], B.dq_ckpt_load(norm.x).double()
    assert torch.equal(xv, P.held(x))
    wants = P.layer_norm_grad(dy, xv, norm.mean, norm.rstd, p["weight"])
    bounds = P.layer_norm_grad_bounds(dy, xv, norm.mean, norm.rstd, p["weight"], dtype, dtype)
    within(g["weight"], wants[1], bounds[1], "weight")
    within(g["bias"], wants[2], bounds[2], "bias")
    # x's gradient is the sum of two, one of them as rounded above: exactly
    assert torch.equal(dx, dout + B.dq_layer_norm_grad(dy, norm, p["weight"])[0])
    # the places between the tensors are left as they were
    assert int((bucket == 5).sum()) >= bucket.numel() - sum(v.numel() for v in g.values())
    # a second micro-batch adds up: the first's values, and the same sums again in binary32, rounded once
    first = {k: v.clone() for k, v in g.items()}
    b.backward(dout, (norm, sy, gate, sh), bucket, accumulate=True)
    if dtype == torch.float32:
        for k, v in b.views(bucket).items():
            assert torch.equal(v, 2 * first[k]), k


def test_workers_buckets_go_through_the_all_reduce(dev):
    """Buckets of whole super-groups for every worker; the sum within what 16-bit widths round (2^-8 of an entry at each of the hops)."""
    n, b = 4, block.Block(64, 96, torch.bfloat16, device=dev)
    buckets, lost = block.worker_gradients(b, n, 100)
    assert len(buckets) == n and all(g.numel() == b.bucket_entries(n) and g.numel() % (n * 256) == 0 and bool(torch.isfinite(g).all()) for g in buckets)
    assert 0 < lost < 2.0 ** -8                          # vNMSE of values off by 2^-4 of themselves at most
    total, info = A.simulated_allreduce(buckets, 17.0, max_width=16, seed=1)
    assert A.vnmse(total, A.true_sum(buckets)) < (n * 2.0 ** -8) ** 2
    assert torch.equal(buckets[0], block.worker_gradients(b, n, 100)[0][0])      # the same bits each time


def test_the_command(dev):
    got = subprocess.run([sys.executable, "-m", "paper_2602_08923_amd.ablation", "--block", "--workers", "2", "--width", "64", "--tokens", "64"],
                         cwd=ROOT, capture_output=True, text=True, timeout=110)
    assert got.returncode == 0, got.stderr[-2000:]
    told = json.loads(got.stdout)
    assert set(told["vNMSE"]) == {"gradients of a feed-forward block"} and 0 < told["vNMSE_of_8_bit_checkpoints"] < 1
