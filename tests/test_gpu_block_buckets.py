"""What a backward pass leaves in its bucket: the places between tensors untouched, a second micro-batch added, a captured one added once more by
each replay."""
import pytest
import torch

from paper_2602_08923_amd import binding as B
from paper_2602_08923_amd import block
from tests import plain_activations as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d,f,rows", [(33, 17, 65), (100, 130, 200)])
def test_a_second_micro_batch_is_added_and_nothing_else_is_written(dev, d, f, rows, dtype):
    b = block.Block(d, f, dtype, seed=3, device=dev)
    x, target = block.tokens(d, rows, 0, dtype, device=dev)
    out, saved = b.forward(x)
    bucket = torch.full((b.bucket_entries(4),), 5.0, dtype=dtype, device=dev)
    between = torch.ones_like(bucket, dtype=torch.bool)
    for v in b.views(between).values():
        v.fill_(False)
    assert int(between.sum()) == bucket.numel() - sum(p.numel() for p in b.params.values()) > 0
    b.backward(out - target, saved, bucket)
    assert bool((bucket[between] == 5).all())
    first = bucket.clone()
    b.backward(out - target, saved, bucket, accumulate=True)
    assert bool((bucket[between] == 5).all())
    # first is the sum s in binary32, rounded; bucket is first + s in binary32, rounded
    one, two, h = first.double()[~between], bucket.double()[~between], P.half_step(dtype)
    s = one.abs() * (1 + 2 * h)
    assert bool(((two - 2 * one).abs() <= s * h + (one.abs() + s) * (h + P.U) * (1 + h) + 1e-37).all())
    assert bool((two != one)[one != 0].all())


def test_replays_add_weight_gradients(dev):
    """Whole numbers under statistics of zero and one (n is x): each replay adds the same sums once more, exactly."""
    rows, cols = 5000, 90
    g = torch.Generator(device=dev).manual_seed(1)
    x, dy = [torch.randint(-3, 4, (rows, cols), generator=g, device=dev).to(torch.bfloat16) for _ in range(2)]
    saved = B.SavedNorm(B.dq_ckpt_save(x), torch.zeros(rows, device=dev), torch.ones(rows, device=dev))
    weight = torch.ones(cols, device=dev)
    want, want_b = (x.double() * dy.double()).sum(0), dy.double().sum(0)
    dw, db = torch.zeros(cols, device=dev), torch.zeros(cols, device=dev)

    def step():
        B.dq_layer_norm_grad(dy, saved, weight, weight_out=dw, bias_out=db, accumulate=True)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for times in range(2, 6):
        graph.replay()
        other = B.dq_layer_norm_grad(dy.flip(0), saved, weight)           # the program's own work between replays
        torch.cuda.synchronize()
        assert torch.equal(dw.double(), times * want) and torch.equal(db.double(), times * want_b), times
        assert torch.equal(other[2].double(), want_b)
