"""Layer norm with a bias and no weight: the bias's gradient."""
import pytest
import torch

from paper_2602_08923_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (300, 515), (70, 20000), (0, 40)])
def test_bias_without_a_weight(dev, rows, cols, dtype):
    g = torch.Generator(device=dev).manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=g, device=dev).to(dtype)
    dy = torch.randint(-9, 10, (rows, cols), generator=g, device=dev).to(dtype)      # sums of whole numbers: exact
    want = dy.double().sum(0)
    b16 = torch.ones(cols, dtype=torch.bfloat16, device=dev)
    y, saved = B.dq_layer_norm(x, bias=b16, save=True)
    dx, dw, none = B.dq_layer_norm_grad(dy, saved)
    assert dw is None and none is None
    got, dw, db = B.dq_layer_norm_grad(dy, saved, bias=True)
    assert dw is None and db.dtype == dtype and torch.equal(db, want.to(dtype)) and torch.equal(got, dx)
    for t in (torch.float32, torch.bfloat16):
        held = torch.full((cols,), 3.0, dtype=t, device=dev)
        got, dw, db = B.dq_layer_norm_grad(dy, saved, bias_out=held)
        assert dw is None and db is held and torch.equal(held, want.to(t)) and torch.equal(got, dx)
        held.fill_(3.0)
        B.dq_layer_norm_grad(dy, saved, bias_out=held, accumulate=True)
        assert torch.equal(held, (want + 3).to(t))


def test_refusals(dev):
    x = torch.randn(6, 64, device=dev)
    _, saved = B.dq_layer_norm(x, save=True)
    w = torch.ones(64, device=dev)
    for call, match in [
        (lambda: B.dq_layer_norm_grad(x, saved, accumulate=True), "without a weight"),
        (lambda: B.dq_layer_norm_grad(x, saved, weight_out=w, bias=True), "without a weight"),
        (lambda: B.dq_layer_norm_grad(x, saved, bias=True, accumulate=True), "give them"),
        (lambda: B.dq_layer_norm_grad(x, saved, bias_out=w[:63]), "bias_out"),
        (lambda: B.dq_layer_norm_grad(x, saved, bias_out=w.half()), "float32 or bfloat16"),
        (lambda: B.dq_layer_norm_grad(x, saved, bias_out=w.cpu()), "different devices"),
        (lambda: B.dq_layer_norm_grad(x, saved, out=w.new_empty(6, 64), bias_out=saved.mean), "bias_out"),
    ]:
        with pytest.raises(B.DqError, match=match):
            call()
