"""The training operators where inputs are not finite, matrices are wide, documents many: what the formulas say there, and refusals that only a device can show."""
import os
import sys

import numpy as np
import pytest
import torch

from gpu_util import DEV, bytes_buffer, dev, host
from oracle import objective, train
from paper_2509_06040_amd import binding as br
from paper_2509_06040_amd import synth
from test_gpu_train_ops import Packed, objective_case

pytestmark = pytest.mark.gpu
FORMS = [("bf16", 64), ("bf16", 128), ("f32", 16), ("f32", 64), ("f32", 128)]


def off_by(got, ref):
    return np.linalg.norm(got - ref) / np.linalg.norm(ref)


# ------------------------------------------------------------------------------------------------------------ attention
@pytest.mark.parametrize("dtype,d", FORMS)
@pytest.mark.parametrize("heads,kv_heads,lq,lk", [(2, 2, (37,), (50,)), (2, 1, (64, 1), (20, 33)), (4, 2, (1201,), (70,)), (1, 1, (3, 130), (700, 5)), (8, 8, (2500,), (300,))])
def test_keys_of_minus_infinity_have_gradients_of_zero(dtype, d, heads, kv_heads, lq, lk):
    """Such keys count as none (probability 0): their dk and dv are 0, and those of the others are as without them, whatever the number of queries.  bf16 rounds the
    terms of a sum twice (P or dS, and the output in dout . out) and the result once, by 0.00166 of a value each in the mean; errors of terms add up as the root of
    their squares, which is above the sum itself where terms cancel; a fifth for the spread.  fp32: sums of up to 2500 terms, 2^-24 of their magnitudes each at most,
    these 30 times the result: 1e-4 has a margin."""
    p = Packed(dtype, d, heads, kv_heads, lq, lk, seed=d + lq[0], front=2, back=3)
    p.q[:] = p.q.abs() + 0.01
    none = np.arange(int(p.k_off[0]), int(p.k_off[-1]), 3)[1:]
    p.k[torch.from_numpy(none).to(DEV)] = -float("inf")
    p.forward()
    p.backward()
    dk, dv = host(p.dk), host(p.dv)
    assert np.all(dk[none] == 0) and np.all(dv[none] == 0)
    q, k, v, do = (host(t).astype(np.float64) for t in (p.q, p.k, p.v, p.dout))
    there = np.setdiff1d(np.arange(len(k)), none)
    k, v, k_off = k[there], v[there], np.searchsorted(there, p.k_off)
    (_, rk, rv), _ = train.attention_grad(do, q, k, v, p.q_off, k_off, p.scale)
    out, _, kept = train.attention(q, k, v, p.q_off, k_off, p.scale)
    squares = np.zeros((2, *k.shape))
    for a, b, x, y, h, pr in kept:
        g = h // (heads // kv_heads)
        ds = pr * (do[a:b, h] @ v[x:y, g].T - (do[a:b, h] * out[a:b, h]).sum(1, keepdims=True)) * p.scale
        squares[0, x:y, g] += (ds ** 2).T @ q[a:b, h] ** 2
        squares[1, x:y, g] += (pr ** 2).T @ do[a:b, h] ** 2
    for got, ref, sq in ((dk, rk, squares[0]), (dv, rv, squares[1])):
        bound = 1.2 * 0.00166 * np.sqrt(2 * sq.sum() + (ref ** 2).sum()) if dtype == "bf16" else 1e-4 * np.linalg.norm(ref)
        assert np.linalg.norm(got[there] - ref) < bound


@pytest.mark.parametrize("dtype,d", FORMS)
@pytest.mark.parametrize("lq", [(1,), (45,), (300,)])
def test_documents_whose_keys_are_all_minus_infinity_have_no_gradients(dtype, d, lq):
    p = Packed(dtype, d, 2, 1, lq, (77,), seed=2)
    p.q[:] = p.q.abs() + 0.01
    p.k[:] = -float("inf")
    p.forward()
    p.backward()
    assert np.all(host(p.out) == 0) and np.all(host(p.dk) == 0) and np.all(host(p.dv) == 0)


# ------------------------------------------------------------------------------------------------------------ objective
@pytest.mark.parametrize("T,splits,K,trees,D", [(8, (2, 4), 2, 1, 64), (8, (2, 4), 2, 2, 8192)])
def test_a_velocity_that_is_not_a_number_shows_in_the_objective(T, splits, K, trees, D):
    """One launch or two: J, the row's log-densities and its gradient are NaN, the other rows' are as they were."""
    c = objective_case(T, splits, K, trees, D, 0.9, True, 0.2, seed=D, moved=0.02)
    c["vd"][1, 5] = float("nan")
    J, new, grad, clipped = torch.zeros(1, device=DEV), torch.empty(c["E"], device=DEV), torch.empty_like(c["vd"]), torch.full((c["E"],), 7, dtype=torch.uint8, device=DEV)
    br.grpo_backward(c["zd"], c["vd"], *c["tables"], dev(c["old"]), dev(c["advn"]), c["clip"], J, new, grad, c["ws"], clipped=clipped)
    hit = np.arange(c["first"][1], c["first"][2])
    rest = np.delete(np.arange(c["R"]), 1)
    assert np.isnan(host(new)[hit]).all() and np.isfinite(np.delete(host(new), hit)).all() and np.all(host(clipped)[hit] == 0)
    assert np.isnan(host(grad)[1]).all() and np.array_equal(host(grad)[rest], c["grad"][rest])
    assert np.isnan(host(J)[0])


def test_a_log_density_that_is_not_a_number_shows_in_the_objectives_value():
    n = 300
    r = np.random.default_rng(0)
    new, old, adv = (r.standard_normal(n).astype(np.float32) for _ in range(3))
    new[17] = np.nan
    J, clipped = torch.zeros(1, device=DEV), torch.full((n,), 7, dtype=torch.uint8, device=DEV)
    br.grpo_objective(dev(new), dev(old), dev(adv), dev(np.arange(n, dtype=np.int32)), n, 0.2, J, clipped)
    ref, marks = objective.grpo_objective(new, old, adv, float(np.float32(0.2)))
    assert np.isnan(ref) and np.isnan(host(J)[0]) and np.array_equal(host(clipped).astype(bool), marks)


# ---------------------------------------------------------------------------------------------------------------- AdamW
def test_adamw_refuses_to_have_its_random_rounding_captured():
    """A replay would draw the captured step's random bits again: elements with low ones would never reach the next code."""
    n = 1000
    p, g = torch.ones(n, device=DEV), torch.full((n,), 0.01, device=DEV)
    m, v, ms, vs = (torch.zeros(k, dtype=t, device=DEV) for k, t in ((n, torch.uint8), (n, torch.uint8), (4, torch.float32), (4, torch.float32)))
    opt = br.AdamW([p], [g], [m], [v], [ms], [vs])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.add_(0.01)
        with pytest.raises(br.BranchRolloutError) as e:
            opt.step()
    assert e.value.code == -1 and "captur" in str(e.value) and opt.cfg.step == 0
    graph.replay()
    torch.cuda.synchronize()
    assert np.all(host(p) == 1) and np.all(host(m) == 0)
    opt.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        opt.step()
    side.synchronize()
    assert opt.cfg.step == 2 and np.all(host(p) < 1) and np.any(host(m) != 0)


# -------------------------------------------------------------------------------------------------------------- example
def test_second_derivatives_are_refused():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import policy_update as example
    off, group = dev(np.array([0, 20, 32], np.int32)), dev(np.array([0, 1], np.int32))
    qkv = torch.randn(32, 3, 2, 16, device=DEV, requires_grad=True)
    x, mods = torch.randn(32, 64, device=DEV, requires_grad=True), torch.randn(2, 2, 64, device=DEV, requires_grad=True)
    for out, leaf in ((example.Attention.apply(qkv, off), qkv), (example.Norm.apply(x, mods, 0, 1, off, group, torch.float32)[0], x)):
        out = out.square().sum()
        first, = torch.autograd.grad(out, leaf, create_graph=True)
        with pytest.raises(RuntimeError, match="differentiate twice"):
            (out + first.square().sum()).backward()


# ---------------------------------------------------------------------------------------------- matrices of 4 GiB and more
class Wide(Packed):
    """Queries, keys, values, output and all gradients as columns of one matrix whose tokens lie `stride` elements apart."""

    def __init__(self, d, heads, kv_heads, lens, stride, seed=0):
        super().__init__("bf16", d, heads, kv_heads, lens, lens, seed=seed)
        T, at, whole = int(self.q_off[-1]), [0], torch.empty(int(self.q_off[-1]) * stride, dtype=torch.bfloat16, device=DEV)

        def column(x):
            n = x.shape[1]
            t = whole.as_strided((T, n, d), (stride, d, 1), at[0])
            t.copy_(x)
            at[0] += n * d
            return t
        for name in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
            setattr(self, name, column(getattr(self, name)))
        self.whole = ()
        self.work = bytes_buffer(max(br.attention_workspace_bytes(self.q, self.k, self.v, self.qo, self.ko, b) for b in (False, True)))


@pytest.mark.parametrize("d,heads,kv_heads", [(64, 2, 2), (128, 2, 1)])
@pytest.mark.parametrize("lens", [(63,), (64,), (33, 0, 31), (1, 70, 60)])
def test_attention_over_matrices_around_4_gib(d, heads, kv_heads, lens):
    """Tokens 64 MiB apart: 63 of them end below 2^32 bytes, 64 do not."""
    Wide(d, heads, kv_heads, lens, 1 << 25, seed=d).run()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("most", [2, 4, 9, 33])
def test_gradients_of_short_documents_of_matrices_past_4_gib_carry_two_roundings(d, most):
    """As in matrices below 4 GiB: 0.00166 sqrt(2) = 0.00235 of the norm; the output's own rounding must not come on top."""
    r = np.random.default_rng(most)
    lens = [int(n) for n in r.integers(2, most + 1, 60)]
    p = Wide(d, 4, 4, lens, ((1 << 31) // sum(lens) // 4096 + 1) * 4096, seed=d + most).run()
    span = p.q.stride(0) * p.q.shape[0] * 2
    assert span >= 1 << 32
    q, k, v, do = (host(t) for t in (p.q, p.k, p.v, p.dout))
    refs, _ = train.attention_grad(do, q, k, v, p.q_off, p.k_off, p.scale)
    for t, ref in zip((p.dq, p.dk, p.dv), refs):
        assert off_by(host(t), ref) < 0.0027


@pytest.mark.parametrize("d", [64, 128])
def test_keys_of_minus_infinity_in_matrices_past_4_gib(d):
    p = Wide(d, 2, 1, (70, 31), 1 << 25, seed=3)
    p.q[:] = p.q.abs() + 0.01
    p.k[::5] = -float("inf")
    p.forward()
    p.backward()
    none = np.arange(101) % 5 == 0
    for t in (p.dk, p.dv):
        assert np.all(host(t)[none] == 0) and np.all(np.isfinite(host(t))) and np.all(host(t)[~none].any((1, 2)))
    assert np.isfinite(host(p.out)).all()
