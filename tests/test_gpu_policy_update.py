"""The example of a policy iteration with its update: its network is the library's, gradients of a parameter are slopes of the objective, updates raise the
objective, and what they write is what the library reads."""
import os
import sys

import numpy as np
import pytest
import torch

from gpu_util import host, rel_l2
from oracle import train
from paper_2509_06040_amd import binding as br
from paper_2509_06040_amd import synth

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import policy_update as example  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("net,tol", [("tiny", 1e-4), ("small", 2e-2)])
def test_the_training_forward_is_the_librarys_network(net, tol):
    """The bars of the library's own velocity against the oracle: 1e-4 in fp32, 2e-2 in bf16."""
    p = example.Policy(example.NETS[net])
    it = example.Iteration(p)
    z, cond = it.z[:6].contiguous(), it.cond
    index = [0, 1, 0, 1, 0, 1]
    want = torch.empty_like(z)
    br.velocity(p.model, z, 0.375, cond, index, want, it.work)
    got = p.velocity(z, torch.full((6,), 0.375, device="cuda"), cond[index])
    assert rel_l2(host(got), host(want)) < tol


@pytest.mark.parametrize("net,bits", [("tiny", 32), ("tiny", 8), ("small", 32), ("small", 8)])
def test_updates_raise_the_objective_and_the_library_sees_them(net, bits):
    p = example.Policy(example.NETS[net], state_bits=bits)
    it = example.Iteration(p)
    # with a clip that does not bite, each small step along the gradient raises J
    values = [float(it.update(p, clip=0.5)) for _ in range(5)]
    assert all(b > a for a, b in zip(values, values[1:])), values
    # log-densities of the next update's forward are those of the library's network with the same weights
    it.update(p, clip=0.5)
    before = host(it.logp_new).copy()
    q = example.Policy(example.NETS[net], state_bits=bits)
    it2 = example.Iteration(q)
    for _ in range(5):
        it2.update(q, clip=0.5)
    lp = torch.empty(len(it2.host_ids), device="cuda")
    br.logprob(it2.tree, q.model, it2.sched, it2.cond, it2.z, it2.host_ids, lp, it2.work)
    assert np.abs(host(lp) - before).max() < (1e-4 if net == "tiny" else 2e-2)


def test_parameter_gradients_are_slopes_of_the_objective():
    """fp32: J along the direction of one tensor's gradient, for tensors on every path: through the norms' vectors, the attention, the stream.  J is taken from the
    velocities in 64 bits; a step moves it by 1e-3, or the tensor by a fiftieth of its norm where that is less: curvature and the velocities' fp32 rounding
    leave 2 % of the slope."""
    p = example.Policy(example.NETS["tiny"])
    it = example.Iteration(p)
    tables = [host(t) for t in it.tables]
    velocity = lambda: p.velocity(it.z[it.tables[1].long()], it.t, it.cond[it.of_tree])  # noqa: E731
    value = lambda v: train.objective_grad(host(it.z), host(v.detach()), *tables, host(it.logp_old), host(it.adv), 0.5, len(tables[0]))[0]  # noqa: E731
    v = velocity()
    grad, room = torch.empty_like(v), torch.empty(br.grpo_backward_workspace_bytes(it.z, v.detach(), *it.tables), dtype=torch.uint8, device="cuda")
    br.grpo_backward(it.z, v.detach(), *it.tables, it.logp_old, it.adv, 0.5, it.J, it.logp_new, grad, room)
    v.backward(grad)
    for name in ("ada_w", "qkv_w", "qkv_b", "fc1_w", "patch_w", "t1_w", "cond_w", "final_w"):
        w, g = p.W[name].detach(), p.W[name].grad
        d = g / g.norm()
        h, f = min(1e-3 / float(g.norm()), float(w.norm()) / 50), []
        for sign in (1, -1):
            w.add_(d, alpha=sign * h)
            with torch.no_grad():
                f.append(value(velocity()))
            w.add_(d, alpha=-sign * h)
        assert abs(-(f[0] - f[1]) / (2 * h) / float(g.norm()) - 1) < 0.02, (name, f)


def test_states_are_the_seeded_ones():
    """Two runs from the same seed give the same parameters, bit for bit (rounding to 8 bits draws from the seed; every operator sums in a fixed order, and so do
    the library products at these sizes)."""
    weights = []
    for _ in range(2):
        p = example.Policy(example.NETS["small"], state_bits=8)
        it = example.Iteration(p)
        for _ in range(3):
            it.update(p)
        weights.append({n: host(p.W[n].detach()).copy() for n in p.names})
    assert synth.SAMPLER_SEED and all(np.array_equal(weights[0][n], weights[1][n]) for n in weights[0])
