"""Forward-mode differentiation has no formulas here: a tensor that carries a tangent is refused, before its device is looked at."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2307_02047_b200 import binding

X, W, IDS = torch.randn(4, 8), torch.randn(8), torch.zeros(3, dtype=torch.int64)
CALLS = [
    ("x", X, lambda t: binding.layer_norm(t)), ("weight", W, lambda t: binding.layer_norm(X, t, W)), ("bias", W, lambda t: binding.layer_norm(X, W, t)),
    ("x of the forward alone", X, lambda t: binding.layer_norm_forward(t)), ("weight of the forward alone", W, lambda t: binding.layer_norm_forward(X, t)),
    ("table of biases", X, lambda t: binding.position_bias_forward(t, 3, 3)), ("table of embeddings", X, lambda t: binding.embed_forward(t, IDS)),
    # gradients of gradients: what reaches a backward pass carries the tangent
    ("gradient of a layer norm", X, lambda t: binding.layer_norm_backward(t, X, W[:4], W[:4])),
    ("gradient of biases", X, lambda t: binding.position_bias_backward(t.view(2, 4, 4), torch.zeros(32, 2))),
    ("gradient of a lookup", X, lambda t: binding.embed_backward(t[:3], IDS, torch.zeros(5, 8))),
]


@pytest.mark.parametrize("name,primal,call", CALLS, ids=[c[0] for c in CALLS])
@pytest.mark.parametrize("requires_grad", [False, True])
def test_a_tangent_is_refused(name, primal, call, requires_grad):
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(primal.clone().requires_grad_(requires_grad), torch.ones_like(primal))
        with pytest.raises(binding.CameError) as e:
            call(dual)
        assert e.value.status == 11 and "forward" in str(e.value)
        # without a tangent the call goes on, to the missing GPU
        with pytest.raises(binding.CameError) as e:
            call(primal)
        assert e.value.status == 7


@pytest.mark.parametrize("name,primal,call", CALLS, ids=[c[0] for c in CALLS])
def test_jvp_is_refused(name, primal, call):
    with pytest.raises(binding.CameError) as e:
        torch.func.jvp(call, (primal,), (torch.ones_like(primal),))
    assert e.value.status == 11
