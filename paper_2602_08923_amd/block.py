"""Gradients from a backward pass: a pre-norm gated feed-forward block, trained data-parallel.

    out = x + down(silu(a) * b),   (a, b) = up(norm(x))

What the backward pass needs of the activations waits in 8-bit checkpoints (the layer norm's input and output, both inputs of the
activation and its output: 8.25 bits an entry each), and every worker's gradients go straight into one flat bucket, each tensor from a
super-group's start on, which is what the all-reduce takes.  The forward products, and those that carry the gradient from layer to
layer, are the library's matrix products; everything else runs in this library's kernels."""
import torch

from . import allreduce as A
from . import binding as B

S = 256  # super-group size


class Block:
    """Parameters of one block of width d and inner width f, all of one dtype (float32 or bfloat16)."""

    def __init__(self, d, f, dtype=torch.bfloat16, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(8_000_000 + seed)

        def normal(*shape):
            return torch.randn(*shape, generator=g, device=device)

        self.d, self.f, self.dtype = d, f, dtype
        self.params = {
            "up": (normal(2 * f, d) / d ** 0.5).to(dtype),
            "down": (normal(d, f) / f ** 0.5).to(dtype),
            "weight": (1.0 + 0.1 * normal(d)).to(dtype),
            "bias": (0.1 * normal(d)).to(dtype),
        }

    def bucket_entries(self, n_workers=1):
        """Entries of a gradient bucket: every tensor from a super-group's start, the whole a multiple of n_workers super-groups."""
        sgs = sum(-(-p.numel() // S) for p in self.params.values())
        return -(-sgs // n_workers) * n_workers * S

    def views(self, bucket):
        """The gradients of the parameters inside a bucket."""
        out, at = {}, 0
        for name, p in self.params.items():
            out[name] = bucket[at:at + p.numel()].view(p.shape)
            at += -(-p.numel() // S) * S
        return out

    def forward(self, x):
        """x: [tokens, d] -> (out, what backward takes)."""
        p, f = self.params, self.f
        y, norm = B.dq_layer_norm(x, p["weight"], p["bias"], save=True)
        saved_y = B.dq_ckpt_save(y)
        ab = y @ p["up"].t()
        h, gate = B.dq_gate(ab[:, :f], ab[:, f:], "silu", save=True)
        saved_h = B.dq_ckpt_save(h)
        return x + h @ p["down"].t(), (norm, saved_y, gate, saved_h)

    def backward(self, dout, saved, bucket, accumulate=False):
        """The gradients of the parameters go to the bucket (accumulate: are added there); returns x's."""
        p, g, f = self.params, self.views(bucket), self.f
        norm, saved_y, gate, saved_h = saved
        B.dq_ckpt_weight_grad(dout, saved_h, out=g["down"], accumulate=accumulate)
        dab = torch.empty(dout.shape[0], 2 * f, dtype=dout.dtype, device=dout.device)
        B.dq_gate_grad(dout @ p["down"], gate, z_out=dab[:, :f], u_out=dab[:, f:])
        B.dq_ckpt_weight_grad(dab, saved_y, out=g["up"], accumulate=accumulate)
        dx, _, _ = B.dq_layer_norm_grad(dab @ p["up"], norm, p["weight"], weight_out=g["weight"], bias_out=g["bias"], accumulate=accumulate)
        return dout + dx

    def plain_gradients(self, x, dout):
        """The same gradients with all activations kept whole, in float32, by PyTorch alone: what the checkpoints are measured against."""
        q = {k: v.detach().float().requires_grad_() for k, v in self.params.items()}
        xf = x.float()
        y = (xf - xf.mean(1, keepdim=True)) * torch.rsqrt(xf.var(1, unbiased=False, keepdim=True) + 1e-5) * q["weight"] + q["bias"]
        a, b = (y @ q["up"].t()).split(self.f, dim=1)
        out = xf + (a * torch.sigmoid(a) * b) @ q["down"].t()
        return dict(zip(q, torch.autograd.grad(out, list(q.values()), dout.float())))


def tokens(d, rows, worker, dtype, seed=0, device="cuda"):
    """A worker's inputs and targets: tokens of different sizes, the targets a fixed rotation of the inputs with noise."""
    g = torch.Generator(device=device)
    g.manual_seed(8_100_000 + 100_000 * seed + worker)
    x = torch.randn(rows, d, generator=g, device=device) * torch.exp(0.5 * torch.randn(rows, 1, generator=g, device=device))
    return x.to(dtype), (x.roll(1, 1) + 0.1 * torch.randn(rows, d, generator=g, device=device)).to(dtype)


def worker_gradients(block, n_workers, rows, micro_batches=2, seed=0):
    """One bucket per worker: gradients of the mean squared error over its own tokens, taken in micro-batches that add up in the bucket.
    Returns (buckets, the error that the 8-bit checkpoints leave in the first worker's, as vNMSE)."""
    buckets, lost = [], None
    dev = block.params["up"].device
    for w in range(n_workers):
        bucket = torch.zeros(block.bucket_entries(n_workers), dtype=block.dtype, device=dev)
        whole = None
        for m in range(micro_batches):
            x, target = tokens(block.d, rows, w * micro_batches + m, block.dtype, seed, dev)
            out, saved = block.forward(x)
            dout = (out - target) * (2.0 / (rows * micro_batches * block.d))
            block.backward(dout, saved, bucket, accumulate=m > 0)
            if w == 0:
                g = block.plain_gradients(x, dout)
                whole = g if whole is None else {k: whole[k] + g[k] for k in g}
        if w == 0:
            flat = torch.zeros_like(bucket, dtype=torch.float32)
            for k, v in block.views(flat).items():
                v.copy_(whole[k])
            lost = A.vnmse(bucket, flat)
        buckets.append(bucket)
    return buckets, lost
