"""The 8-bit activation checkpoints and the passes that write and read them, as cases that can be timed and compared.

What stands behind the list: a data-parallel training job whose gradients this library carries keeps what its backward pass needs in
8-bit blocks (32 entries along a row share a power of two), and its backward pass reads them: the weight gradient of a linear layer,
layer norm, the activation between two linear layers.  Widths 2048, 6144 and 8192 are those of the table of shapes in workloads.py.

`own` False: the operators in elementary torch operations.  True: the library's calls.
"""
import math

import torch

own = False

BLOCK = 32
LOWEST, HIGHEST = 10, 246        # scale exponents (biased by 127): every value is a normal bfloat16 or zero
EPS = 1e-5


def _checkpoint(rows, cols, dtype, parts):
    """Save a tensor and read it back.  parts: the tensor is one of so many side by side, as of a fused projection."""
    return {"op": "checkpoint", "rows": rows, "cols": cols, "dtype": dtype, "parts": parts}


def _weight_grad(rows, outs, cols, dtype, bias):
    """The weight gradient of a linear layer cols -> outs over so many tokens, its input from a checkpoint."""
    return {"op": "weight_grad", "rows": rows, "outs": outs, "cols": cols, "dtype": dtype, "bias": bias}


def _layer_norm(rows, cols, dtype, weights, train):
    """Layer norm: train: the forward pass with its checkpoint and the backward pass from it; else the forward pass alone."""
    return {"op": "layer_norm", "rows": rows, "cols": cols, "dtype": dtype, "weights": weights, "train": train}


def _gate(rows, cols, dtype, kind, gated, train):
    """act(z) or act(z) * u, forward and from checkpoints backward (train), z and u side by side in one projection's output."""
    return {"op": "gate", "rows": rows, "cols": cols, "dtype": dtype, "kind": kind, "gated": gated, "train": train}


def listed():
    return [
        # one token's activations: the time of a call
        dict(_checkpoint(1, 2048, "bf16", 1), name="checkpoint_1x2048_bf16"),
        # a feed-forward block's inner activations of one micro-batch: the largest tensor that waits for the backward pass
        dict(_checkpoint(16384, 8192, "bf16", 1), name="checkpoint_16384x8192_bf16"),
        # an odd width in fp32, the middle one of three tensors side by side: rows start anywhere, blocks end inside the row
        dict(_checkpoint(4099, 2051, "f32", 3), name="checkpoint_4099x2051_f32"),
        # a handful of tokens (a ragged last micro-batch), odd width out: writing the gradient is all there is
        dict(_weight_grad(5, 515, 2048, "bf16", True), name="weight_grad_5x515x2048_bf16"),
        # an attention output projection over a micro-batch of 8,192 tokens
        dict(_weight_grad(8192, 2048, 2048, "bf16", False), name="weight_grad_8192x2048x2048_bf16"),
        # a feed-forward projection over 16,384 tokens, with its bias: the largest products
        dict(_weight_grad(16384, 8192, 2048, "bf16", True), name="weight_grad_16384x8192x2048"),
        # many tokens and a small layer in fp32: the sum over tokens is all there is to share out
        dict(_weight_grad(65537, 200, 136, "f32", True), name="weight_grad_65537x200x136_f32"),
        # one token, forward alone, as a model answers
        dict(_layer_norm(1, 2048, "bf16", "bf16", False), name="layer_norm_1x2048_bf16"),
        # a training step over a micro-batch of 16,384 tokens, weights in fp32
        dict(_layer_norm(16384, 2048, "bf16", "f32", True), name="layer_norm_16384x2048_bf16"),
        # a wide odd row in fp32
        dict(_layer_norm(1021, 6151, "f32", "f32", True), name="layer_norm_1021x6151_f32"),
        # the gated activation of a training step
        dict(_gate(16384, 8192, "bf16", "silu", True, True), name="gate_16384x8192_bf16"),
        # a small ungated one in fp32
        dict(_gate(33, 1000, "f32", "gelu", False, True), name="gate_33x1000_f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["checkpoint", "weight_grad", "weight_grad", "layer_norm", "layer_norm", "gate"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    cols = _log(rng, 16, 8192)
    if rng.random() < 0.5:                     # widths are multiples of 64 as often as anything
        cols = max(64, cols // 64 * 64)
    if op == "weight_grad":
        outs = _log(rng, 16, 8192)
        if rng.random() < 0.5:
            outs = max(64, outs // 64 * 64)
        return _weight_grad(_log(rng, 1, min(65536, 250_000_000_000 // (outs * cols))), outs, cols, dtype, rng.random() < 0.5)
    rows = _log(rng, 1, min(65536, 100_000_000 // cols))
    if op == "checkpoint":
        return _checkpoint(rows, cols, dtype, rng.choice([1, 1, 3]))
    if op == "layer_norm":
        return _layer_norm(rows, cols, dtype, rng.choice([dtype, "f32"]), rng.random() < 0.75)
    return _gate(rows, cols, dtype, rng.choice(["silu", "gelu"]), rng.random() < 0.7, rng.random() < 0.75)


# ---------------------------------------------------------------------------------------- inputs
def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _activations(g, rows, cols):
    """Tokens of different sizes, a few features far larger than the rest."""
    x = _normal(g, rows, cols)
    x *= torch.exp(0.5 * _normal(g, rows, 1))
    loud = torch.rand(1, cols, generator=g, device="cuda") < 0.01
    x *= torch.where(loud, 30.0, 1.0)
    return x.add_(0.2 * _normal(g, 1, cols))


def prepare(case, seed):
    g = _generator(seed)
    rows, cols, t = case["rows"], case["cols"], _dtype(case["dtype"])
    s = {"op": case["op"]}
    if case["op"] == "checkpoint":
        parts = case["parts"]
        whole = torch.empty(rows, parts * cols, dtype=t, device="cuda")
        for p in range(parts):
            whole[:, p * cols:(p + 1) * cols] = _activations(g, rows, cols)
        s["x"] = whole[:, parts // 2 * cols:(parts // 2 + 1) * cols]
    elif case["op"] == "weight_grad":
        x = _activations(g, rows, cols).to(torch.bfloat16)
        s["checkpoint"], s["cols"] = _checkpoint_bytes(x.float()), cols            # what the forward pass has left
        s["dy"] = (1e-3 * _normal(g, rows, case["outs"])).to(t)
        s["bias"] = case["bias"]
    elif case["op"] == "layer_norm":
        w = _dtype(case["weights"])
        s["x"] = _activations(g, rows, cols).to(t)
        s["weight"] = (1.0 + 0.2 * _normal(g, cols)).to(w)
        s["bias"] = (0.2 * _normal(g, cols)).to(w)
        s["train"] = case["train"]
        if s["train"]:
            s["dy"] = (1e-3 * _normal(g, rows, cols)).to(t)
    else:
        n = 2 if case["gated"] else 1
        both = torch.empty(rows, n * cols, dtype=t, device="cuda")
        for p in range(n):
            both[:, p * cols:(p + 1) * cols] = _activations(g, rows, cols)
        s["z"] = both[:, :cols]
        s["u"] = both[:, cols:] if case["gated"] else None
        s["kind"], s["train"] = case["kind"], case["train"]
        if s["train"]:
            s["dh"] = (1e-3 * _normal(g, rows, cols)).to(t)
    return s


# ---------------------------------------------------------------------------------------- the plain forms
def _blocks(x):
    """x (fp32) in blocks of 32 along a row, each entry rounded to E4M3 in units of its block's power of two, and the powers' exponents."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % BLOCK)).reshape(rows, -1, BLOCK)
    e = (x.abs().amax(dim=2, keepdim=True).view(torch.int32) >> 23) - 8
    e = e.clamp(LOWEST, HIGHEST)
    v = x * ((254 - e) << 23).view(torch.float32)                                  # exact
    step = (((v.abs().view(torch.int32) >> 23).clamp(min=121) - 3) << 23).view(torch.float32)   # between neighbouring codes
    return (torch.round(v / step) * step).clamp(-448.0, 448.0), e                  # ties to even


def _held(x):
    """The values that a checkpoint of x (fp32) stands for."""
    v, e = _blocks(x)
    return (v * (e << 23).view(torch.float32)).reshape(len(x), -1)[:, :x.shape[1]]


def _checkpoint_bytes(x):
    """A checkpoint's bytes: a code an entry (rows filled up to whole blocks), then an exponent a block."""
    v, e = _blocks(x)
    size = v.abs()
    code = torch.where(size < 2.0 ** -6, (size * 512.0).to(torch.int32), (size.view(torch.int32) >> 20) - (120 << 3))
    code += torch.where(torch.signbit(v), 128, 0)
    return torch.cat([code.to(torch.uint8).reshape(-1), e.to(torch.uint8).reshape(-1)])


def _checkpoint_values(data, rows, cols):
    """The values that a checkpoint's bytes stand for, in fp32."""
    wide = cols + -cols % BLOCK
    code = data[:rows * wide].to(torch.int32)
    low = code & 127
    v = torch.where(low < 8, low.float() / 512.0, ((low << 20) + (120 << 23)).view(torch.float32))
    v = torch.where(code > 127, -v, v).reshape(rows, -1, BLOCK)
    return (v * (data[rows * wide:].to(torch.int32) << 23).view(torch.float32).reshape(rows, -1, 1)).reshape(rows, wide)[:, :cols]


def _activation(z, kind):
    """act(z) and its derivative."""
    if kind == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return z * p, p * (1.0 + z * (1.0 - p))
    p = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z * p, p + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_layer_norm(s):
    t, x, w = s["x"].dtype, s["x"].float(), s["weight"].float()
    mean = x.mean(dim=1, keepdim=True)
    rstd = torch.rsqrt((x - mean).square().mean(dim=1, keepdim=True) + EPS)
    y = (((x - mean) * rstd) * w + s["bias"].float()).to(t)
    if not s["train"]:
        return y
    xh = (_held(x) - mean) * rstd
    dy = s["dy"].float()
    q = dy * w
    dx = rstd * (q - q.mean(dim=1, keepdim=True) - xh * (q * xh).mean(dim=1, keepdim=True))
    return [y, dx.to(t), (dy * xh).sum(dim=0).to(s["weight"].dtype), dy.sum(dim=0).to(s["bias"].dtype)]


def _plain_gate(s):
    t, z, u = s["z"].dtype, s["z"].float(), None if s["u"] is None else s["u"].float()
    a, _ = _activation(z, s["kind"])
    h = (a if u is None else a * u).to(t)
    if not s["train"]:
        return h
    a, d = _activation(_held(z), s["kind"])
    dh = s["dh"].float()
    if u is None:
        return [h, (dh * d).to(t)]
    return [h, (dh * _held(u) * d).to(t), (dh * a).to(t)]


def run(s):
    if own:
        return _own(s)
    if s["op"] == "checkpoint":
        return _held(s["x"].float()).to(s["x"].dtype)
    if s["op"] == "weight_grad":
        dy = s["dy"].float()
        dw = (dy.t() @ _checkpoint_values(s["checkpoint"], len(dy), s["cols"])).to(s["dy"].dtype)
        return [dw, dy.sum(dim=0).to(s["dy"].dtype)] if s["bias"] else dw
    return _plain_layer_norm(s) if s["op"] == "layer_norm" else _plain_gate(s)


# ---------------------------------------------------------------------------------------- the library's calls
def _own(s):
    from paper_2602_08923_amd import binding as B
    if s["op"] == "checkpoint":
        return B.dq_ckpt_load(B.dq_ckpt_save(s["x"]), s["x"].dtype)
    if s["op"] == "weight_grad":
        saved = B.Checkpoint(s["checkpoint"], len(s["dy"]), s["cols"])
        return B.dq_ckpt_weight_grad(s["dy"], saved, bias=s["bias"])
    if s["op"] == "layer_norm":
        if not s["train"]:
            return B.dq_layer_norm(s["x"], s["weight"], s["bias"], EPS)
        y, saved = B.dq_layer_norm(s["x"], s["weight"], s["bias"], EPS, save=True)
        return [y, *B.dq_layer_norm_grad(s["dy"], saved, s["weight"])]
    if not s["train"]:
        return B.dq_gate(s["z"], s["u"], s["kind"])
    h, saved = B.dq_gate(s["z"], s["u"], s["kind"], save=True)
    dz, du = B.dq_gate_grad(s["dh"], saved)
    return [h, dz] if du is None else [h, dz, du]


# ---------------------------------------------------------------------------------------- work and exact values
def work(case):
    rows, cols, n = case["rows"], case["cols"], 4 if case["dtype"] == "f32" else 2
    held = rows * cols * 33 / 32
    if case["op"] == "checkpoint":             # in, held and read again, out
        return {"bytes": 2 * n * rows * cols + 2 * held, "flops": 4.0 * rows * cols}
    if case["op"] == "weight_grad":
        outs = case["outs"]
        return {"bytes": n * rows * outs + held + n * outs * (cols + (1 if case["bias"] else 0)), "flops": 2.0 * rows * outs * cols}
    if case["op"] == "layer_norm":
        w = 4 if case["weights"] == "f32" else 2
        if not case["train"]:
            return {"bytes": 2 * n * rows * cols + 2 * w * cols, "flops": 8.0 * rows * cols}
        return {"bytes": 4 * n * rows * cols + 2 * held + 4 * w * cols, "flops": 24.0 * rows * cols}
    k = 2 if case["gated"] else 1
    if not case["train"]:
        return {"bytes": (k + 1) * n * rows * cols, "flops": 10.0 * rows * cols}
    return {"bytes": (2 * k + 2) * n * rows * cols + 2 * k * held, "flops": 30.0 * rows * cols}


def _magnitudes(device):
    """The 127 magnitudes of E4M3, in the order of their codes."""
    m = [m / 8 * 2.0 ** -6 for m in range(8)] + [(1 + m / 8) * 2.0 ** p for p in range(-6, 9) for m in range(8)]
    return torch.tensor(m[:127], dtype=torch.float64, device=device)


def _power(e):
    """2^e in 64 bits."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _nearest(x):
    """The held values of x in 64 bits: each block's power of two from its largest entry, then the nearest of all magnitudes."""
    rows, cols = x.shape
    table = _magnitudes(x.device)
    middles = (table[1:] + table[:-1]) / 2
    out = torch.zeros(rows, cols + -cols % BLOCK, dtype=torch.float64, device=x.device)
    out[:, :cols] = x
    blocks = out.view(-1, BLOCK)
    for part in blocks.split(1 << 20):         # views of out: written in place
        top = torch.frexp(part.abs().amax(dim=1, keepdim=True)).exponent - 1       # floor(log2)
        scale = _power((top - 8).clamp(LOWEST - 127, HIGHEST - 127))
        v = (part / scale).abs()
        below = torch.searchsorted(middles, v, right=False)
        tie = below != torch.searchsorted(middles, v, right=True)
        code = below + torch.where(tie, below % 2, torch.zeros_like(below))         # halfway: the even code
        part.copy_(torch.copysign(table[code], part) * scale)
    return out[:, :cols]


def _read(data, rows, cols):
    """A checkpoint's values in 64 bits, by a table of all codes."""
    wide = cols + -cols % BLOCK
    table = torch.cat([_magnitudes(data.device), torch.full((1,), math.nan, dtype=torch.float64, device=data.device)])
    table = torch.cat([table, -table])
    codes, exponents = data.split([rows * wide, rows * wide // BLOCK])
    out = torch.empty(rows * wide // BLOCK, BLOCK, dtype=torch.float64, device=data.device)
    for to, c, e in zip(out.split(1 << 20), codes.view(-1, BLOCK).split(1 << 20), exponents.split(1 << 20)):
        to.copy_(table[c.to(torch.int64)] * _power(e.to(torch.int64) - 127)[:, None])
    return out.view(rows, wide)[:, :cols]


def _exact_activation(z, kind):
    if kind == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * torch.sigmoid(-z)
    p = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def exact(case, seed):
    s = prepare(case, seed)
    rows, cols = case["rows"], case["cols"]
    if case["op"] == "checkpoint":
        return _nearest(s["x"].double())
    if case["op"] == "weight_grad":
        dy, x = s["dy"].double(), _read(s["checkpoint"], rows, cols)
        dw = torch.zeros(dy.shape[1], x.shape[1], dtype=torch.float64, device=x.device)
        for a, b in zip(dy.split(4096), x.split(4096)):
            dw += a.t().contiguous() @ b
        return [dw, dy.sum(dim=0)] if case["bias"] else dw
    if case["op"] == "layer_norm":
        x, w = s["x"].double(), s["weight"].double()
        mean, var = x.mean(dim=1, keepdim=True), x.var(dim=1, unbiased=False, keepdim=True)
        deviation = torch.sqrt(var + EPS)
        y = (x - mean) / deviation * w + s["bias"].double()
        if not case["train"]:
            return y
        n = (_nearest(x) - mean) / deviation
        dy = s["dy"].double()
        q = dy * w
        dx = (q - q.mean(dim=1, keepdim=True) - n * (q * n).mean(dim=1, keepdim=True)) / deviation
        return [y, dx, (dy * n).sum(dim=0), dy.sum(dim=0)]
    z, u = s["z"].double(), None if s["u"] is None else s["u"].double()
    h = _exact_activation(z, case["kind"])[0] * (1.0 if u is None else u)
    if not case["train"]:
        return h
    a, d = _exact_activation(_nearest(z), case["kind"])
    dh = s["dh"].double()
    return [h, dh * d] if u is None else [h, dh * _nearest(u) * d, dh * a]
