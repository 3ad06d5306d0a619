"""Forward-mode derivatives: the calls propagate no tangents, so a tensor that has one is
refused, as one that requires a gradient is."""
import pytest
import torch
from torch.autograd import forward_ad as F

from paper_2609_34244_amd import heddle as H


def dual(t):
    return F.make_dual(t, torch.ones_like(t))


def test_tensors_with_a_tangent():
    """the checks of the arguments, on tensors of the CPU"""
    t = torch.ones(2, 3, 4, 8, dtype=torch.bfloat16)
    checks = [lambda x: H._heads(x, "q", (2, 3, 4, 8), torch.bfloat16, -1), lambda x: H._matrix(x[0, 0], "x", (4, 8), torch.bfloat16, -1),
              lambda x: H._vector(x[0, 0, 0], "w", (8,), torch.bfloat16, -1), lambda x: H._weights(x[0], "w", (3, 4, 8), torch.bfloat16, -1)]
    for check in checks:
        want = check(t)
        with F.dual_level():
            assert check(t) == want
            for grad in (True, False):
                with torch.set_grad_enabled(grad), pytest.raises(H.HeddleError, match="forward-mode") as e:
                    check(dual(t))
                assert e.value.code == H.HEDDLE_E_INVAL
            with F._set_fwd_grad_enabled(False):
                check(t)
        check(t)


@pytest.mark.gpu
def test_calls():
    def ones(*s, dtype=torch.bfloat16):
        return torch.ones(s, dtype=dtype, device="cuda")

    x, w, q, slopes = ones(4, 8), ones(8, 8), ones(1, 4, 2, 16), ones(2, dtype=torch.float32)
    logits, picked, dloss = ones(4, 8, dtype=torch.float32), torch.zeros(4, 2, dtype=torch.int64, device="cuda"), ones(1, dtype=torch.float32)
    b = H.heddle_expert_balance(logits, picked)
    calls = {"linear": (H.heddle_linear, [x, w]), "norm": (H.heddle_layer_norm, [x, w[0], w[1]]), "attention": (H.heddle_attention, [q, q, q]),
             "slopes": (lambda s: H.heddle_attention(q, q, q, slopes=s), [slopes]), "balance": (lambda z: H.heddle_expert_balance(z, picked)["loss"], [logits]),
             "balance backward": (lambda z, d: H.heddle_expert_balance_backward(z, picked, b["counts"], b["rows"], dloss=d), [logits, dloss])}
    for name, (call, args) in calls.items():
        want = call(*args)
        with F.dual_level():
            assert torch.equal(call(*args), want), name
            for i in range(len(args)):
                with pytest.raises(H.HeddleError, match="forward-mode"):
                    call(*(dual(a) if i == j else a for j, a in enumerate(args)))
