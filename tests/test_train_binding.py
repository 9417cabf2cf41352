"""Checks of the binding in front of the training operators.  No kernel is launched: every call ends at its checks, so host tensors will do."""
import pytest
import torch

from paper_2509_06040_amd import binding as br


def leaf(n, dtype=torch.float32):
    x = torch.ones(n, dtype=dtype, requires_grad=True)
    x.grad = torch.ones(n, dtype=dtype)
    return x


def states(n):
    return torch.zeros(n), torch.zeros(n)


@pytest.mark.parametrize("bf16", [False, True])
def test_adamw_notices_gradients_that_are_other_tensors_now(bf16):
    """A leaf (the parameter, or the copy that the network reads) whose .grad was handed over: set to None and made anew, the optimizer would go on with the old one."""
    x, (m, v) = leaf(10, torch.bfloat16 if bf16 else torch.float32), states(10)
    p, copies = (x.detach().float(), [x]) if bf16 else (x, None)
    opt = br.AdamW([p], [x.grad], [m], [v], copies=copies)
    torch.optim.SGD([x], lr=0.0).zero_grad(set_to_none=True)
    with pytest.raises(ValueError, match="gradient"):
        opt.step()
    x.grad = torch.ones_like(x)
    with pytest.raises(ValueError, match="gradient"):
        opt.step()
    assert opt.cfg.step == 0
