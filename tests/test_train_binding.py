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


@pytest.mark.parametrize("wrong", [torch.ones(1, dtype=torch.float64), torch.ones(1, dtype=torch.bfloat16), torch.ones(0), torch.ones(2), torch.ones(4)[::2][:1].expand(3)])
def test_adamw_takes_one_fp32_factor(wrong):
    m, v = states(10)
    opt = br.AdamW([torch.ones(10)], [torch.ones(10)], [m], [v])
    with pytest.raises(AssertionError):
        opt.step(grad_scale=wrong)
    assert opt.cfg.step == 0


@pytest.mark.parametrize("wrong", [dict(clipped=torch.zeros(3, dtype=torch.int32)), dict(clipped=torch.zeros(2, dtype=torch.uint8)), dict(clipped=torch.zeros(6, dtype=torch.uint8)[::2]),
                                   dict(J=torch.zeros(0)), dict(J=torch.zeros(2)), dict(J=torch.zeros(1, dtype=torch.float64)), dict(logp_new=torch.zeros(2)), dict(adv=torch.zeros(7))])
def test_objective_takes_outputs_of_its_sizes_and_types(wrong):
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32)  # noqa: E731
    t = dict(adv=torch.zeros(8), J=torch.zeros(1), logp_new=torch.zeros(3), clipped=None)
    t.update(wrong)
    with pytest.raises(AssertionError):
        br.grpo_backward(torch.zeros(8, 4), torch.zeros(2, 4), i32(1, 2, 5), i32(0, 3), i32(0, 2, 3), torch.zeros(2, 4, dtype=torch.float64), torch.zeros(8), t["adv"], 0.1, t["J"], t["logp_new"],
                         torch.zeros(2, 4), torch.zeros(1 << 12, dtype=torch.uint8), clipped=t["clipped"])
