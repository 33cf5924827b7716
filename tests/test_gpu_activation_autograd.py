"""The activation operators beside autograd: what they return has no graph, and a tensor that they write to counts as changed in place, so that a
graph that has kept it does not go on with other values."""
import pytest
import torch

from paper_2602_08923_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def test_outputs_given_count_as_changed(dev):
    x, w = torch.randn(6, 64, device=dev), torch.ones(64, device=dev)
    ck = B.dq_ckpt_save(x)
    _, norm = B.dq_layer_norm(x, w, w, save=True)
    _, gate = B.dq_gate(x, x, save=True)
    outs = {k: torch.zeros(6, 64, device=dev) for k in ("load", "norm", "dx", "h", "dz", "du")}
    dw, db, w2, b2 = torch.zeros(64, 64, device=dev), torch.zeros(64, device=dev), torch.zeros(64, device=dev), torch.zeros(64, device=dev)
    data = torch.zeros_like(ck.data)
    given = list(outs.values()) + [dw, db, w2, b2, data]
    before = [t._version for t in given + [x, w]]
    B.dq_ckpt_save(x, data)
    B.dq_ckpt_load(ck, out=outs["load"])
    B.dq_ckpt_weight_grad(x, ck, out=dw, bias_out=db)
    B.dq_layer_norm(x, w, w, out=outs["norm"])
    B.dq_layer_norm_grad(x, norm, w, out=outs["dx"], weight_out=w2, bias_out=b2)
    B.dq_gate(x, x, out=outs["h"])
    B.dq_gate_grad(x, gate, outs["dz"], outs["du"])
    assert [t._version for t in given + [x, w]] == [v + 1 for v in before[:len(given)]] + before[len(given):]
    with torch.inference_mode():
        kept = torch.zeros(6, 64, device=dev)
        B.dq_layer_norm(x, out=kept)
    B.dq_layer_norm(x, out=kept)


def test_a_graph_that_kept_an_output_says_so(dev):
    x = torch.randn(6, 64, device=dev)
    a = torch.randn(6, 64, device=dev, requires_grad=True)
    held = torch.ones(6, 64, device=dev)
    total = (a * held).sum()
    assert not B.dq_layer_norm(a).requires_grad
    B.dq_layer_norm(x, out=held)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        total.backward()
