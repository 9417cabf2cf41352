"""The operators of a policy update against the oracle's 64 bits: lengths around the tiles' edges, empty documents, rows of no document, strides, shared heads,
odd sizes; gradients against differences; side streams, graphs, equal bits on equal inputs."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, bytes_buffer, dev, host
from oracle import train
from paper_2509_06040_amd import binding as br
from paper_2509_06040_amd import synth

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------------------------ attention
class Packed:
    """Inputs of an attention call: queries, keys and values side by side in one buffer of `pad` spare columns (the type's unit), tokens
    in front of the first document and behind the last one."""

    def __init__(self, dtype, d, heads, kv_heads, lq, lk, seed=0, front=0, back=0, size=1.0):
        r = np.random.default_rng(seed)
        self.T, self.dtype, self.d, self.heads, self.kv = TYPES[dtype], dtype, d, heads, kv_heads
        self.q_off, self.k_off = front + np.cumsum((0,) + tuple(lq)), front + np.cumsum((0,) + tuple(lk))
        Tq, Tk = int(self.q_off[-1]) + back, int(self.k_off[-1]) + back
        wide = lambda n, h: dev(r.standard_normal((n, h + 1, d)).astype(np.float32) * size, self.T)
        q, kv = wide(Tq, heads), wide(Tk, 2 * kv_heads)
        self.q, self.k, self.v = q[:, :heads], kv[:, :kv_heads], kv[:, kv_heads:2 * kv_heads]
        self.dout = wide(Tq, heads)[:, :heads]
        self.out, self.lse = torch.full((Tq, heads + 1, d), 7.0, device=DEV).to(self.T)[:, :heads], torch.full((heads, Tq), 7.0, device=DEV)
        dq, dkv = torch.full((Tq, heads + 1, d), 7.0, device=DEV).to(self.T), torch.full((Tk, 2 * kv_heads + 1, d), 7.0, device=DEV).to(self.T)
        self.whole = (dq, dkv)
        self.dq, self.dk, self.dv = dq[:, :heads], dkv[:, :kv_heads], dkv[:, kv_heads:2 * kv_heads]
        self.qo, self.ko = dev(self.q_off.astype(np.int32)), dev(self.k_off.astype(np.int32))
        self.work = bytes_buffer(max(br.attention_workspace_bytes(self.q, self.k, self.v, self.qo, self.ko, b) for b in (False, True)))
        self.scale = float(np.float32(1 / np.sqrt(d)))

    def forward(self, **more):
        br.attention_forward(self.q, self.k, self.v, self.qo, self.ko, self.out, self.lse, self.work, **more)

    def backward(self, **more):
        br.attention_backward(self.dout, self.q, self.k, self.v, self.out, self.lse, self.qo, self.ko, self.dq, self.dk, self.dv, self.work, **more)

    def check(self, scale=None):
        """Tolerances.  A score is a sum of d products in fp32 (d 2^-24 of the sum of their magnitudes at most), its exponential and the normaliser add
        2^-22 of a probability and of the score's own size: e.  bf16 rounds a probability or its gradient once more, the result, and the output that
        enters dout . out: each by 2^-8 of the terms at most (a sum of one term has all of it): 3 * 2^-8 of the sum of their magnitudes."""
        scale = scale or self.scale
        q, k, v, do = (host(t) for t in (self.q, self.k, self.v, self.dout))
        out, lse, _ = train.attention(q, k, v, self.q_off, self.k_off, scale)
        mean, _, _ = train.attention(q, k, np.abs(v), self.q_off, self.k_off, scale)  # sum of p |v|
        most = np.abs(q).max(initial=0) * np.abs(k).max(initial=0) * scale * self.d ** 0.5 * 4
        e = (self.d + 8) * 2.0 ** -24 * most + 2.0 ** -20
        low = 3 * 2.0 ** -8 if self.dtype == "bf16" else 0
        got = host(self.out)
        assert np.all(np.abs(got - out) <= (2 * e + low) * mean), np.max(np.abs(got - out) / np.maximum(mean, 1e-30))
        l = host(self.lse)
        assert np.array_equal(np.isinf(l), np.isinf(lse)) and np.all(l[np.isinf(l)] < 0)
        assert np.all(np.abs(l - lse)[~np.isinf(l)] <= e + 2.0 ** -23 * np.abs(lse[~np.isinf(l)]))
        if self.graded:
            refs, weights = train.attention_grad(do, q, k, v, self.q_off, self.k_off, scale)
            for name, t, ref, w in zip(("dq", "dk", "dv"), (self.dq, self.dk, self.dv), refs, weights):
                g = host(t)
                assert np.all(np.abs(g - ref) <= (4 * e + low) * w + 1e-30), (name, np.max(np.abs(g - ref) / np.maximum(w, 1e-30)))
            for t, n in zip(self.whole, (self.heads, 2 * self.kv)):  # the columns between tokens are not touched
                assert np.all(host(t)[:, n:] == 7.0)

    graded = False

    def run(self, scale=None):
        self.forward(scale=scale)
        self.backward(scale=scale)
        self.graded = True
        self.check(scale)
        return self


LENGTHS = [
    ((1,), (1,)), ((1, 2, 3), (5, 1, 64)), ((63, 64, 65), (63, 64, 65)), ((127, 128, 129, 130), (129, 31, 32, 33)), ((0, 5, 0, 0, 70), (3, 0, 4, 0, 200)),
    ((300,), (17,)), ((3,), (517,)), ((260, 1), (255, 257)), ((16,) * 70, (16,) * 70), ((0,), (9,)), ((9,), (0,)),
]


@pytest.mark.parametrize("lq,lk", LENGTHS)
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 16), ("f32", 32), ("f32", 64), ("f32", 128)])
def test_attention_over_ragged_documents(dtype, d, lq, lk):
    Packed(dtype, d, 2, 2, lq, lk, seed=len(lq) + lq[0]).run()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("heads,kv_heads", [(4, 1), (6, 3), (3, 3)])
def test_attention_shared_heads_and_tokens_of_no_document(dtype, d, heads, kv_heads):
    p = Packed(dtype, d, heads, kv_heads, (70, 0, 130), (40, 3, 200), seed=heads, front=5, back=66).run()
    out, lse = host(p.out), host(p.lse)
    none = np.r_[0:5, p.q_off[-1]:len(out)]
    assert np.all(out[none] == 0) and np.all(lse[:, none] == -np.inf) and np.all(host(p.dq)[none] == 0)
    none = np.r_[0:5, 45:48, p.k_off[-1]:p.k.shape[0]]  # (keys of the document without queries too)
    assert np.all(host(p.dk)[none] == 0) and np.all(host(p.dv)[none] == 0)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 32), ("f32", 64)])
@pytest.mark.parametrize("heads,kv_heads,lq,lk", [(2, 2, (20,), (3000,)), (2, 2, (3000,), (20,)), (8, 2, (700, 0, 650), (700, 33, 650)), (4, 1, (900,), (70,)),
                                                (1, 1, (1, 2000, 1), (2500, 1, 0)), (4, 2, (129, 1500), (1600, 31))])
def test_attention_with_few_rows_on_one_side(dtype, d, heads, kv_heads, lq, lk):
    """Launches that leave units empty: the other side's rows in parts, whose sums a launch behind joins; tokens of no document among them."""
    p = Packed(dtype, d, heads, kv_heads, lq, lk, seed=heads, front=3, back=40).run()
    assert np.all(host(p.out)[:3] == 0) and np.all(host(p.dk)[-40:] == 0) and np.all(host(p.dv)[:3] == 0)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 16)])
@pytest.mark.parametrize("heads", [1, 2, 6, 7, 12, 16])
def test_attention_of_any_number_of_heads_and_many_documents(dtype, d, heads):
    """Heads are dealt to the compute dies in groups of their common divisor with eight; more documents than a wavefront has lanes, empty ones among them."""
    r = np.random.default_rng(heads)
    lens = [int(n) * int(r.random() < 0.8) for n in r.integers(1, 40, 150)] + [140, 0, 260]
    Packed(dtype, d, heads, heads, lens, lens, seed=heads).run()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_attention_where_most_scores_are_minus_infinity(dtype, d):
    """Keys whose products are all -inf count as none, in parts of a document and in whole ones; outputs and probabilities of the others are as without them."""
    p = Packed(dtype, d, 2, 2, (30,), (2000,), seed=3)
    p.q[:] = p.q.abs() + 0.01
    p.k[:1900] = -float("inf")
    p.forward()
    out, lse = host(p.out), host(p.lse)
    q, k, v = (host(t).astype(np.float64) for t in (p.q, p.k, p.v))
    ref, rl, _ = train.attention(q, k[1900:], v[1900:], [0, 30], [0, 100], p.scale)
    assert np.abs(out - ref).max() < (0.03 if dtype == "bf16" else 1e-4) and np.abs(lse - rl).max() < 1e-4
    p.k[:] = -float("inf")
    p.forward()
    assert np.all(host(p.out) == 0) and np.all(host(p.lse) == -np.inf)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 128)])
def test_attention_many_heads_long_documents(dtype, d):
    Packed(dtype, d, 4, 4, (1100, 700), (1100, 700), seed=4).run()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 32)])
def test_attention_with_scores_far_apart(dtype, d):
    """Scores of some hundreds: a maximum that moves at almost every tile, most probabilities zero; another scale."""
    p = Packed(dtype, d, 2, 1, (150, 90), (333, 64), seed=8, size=6.0)
    p.run(scale=0.5)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_attention_keeps_what_is_not_finite_to_its_own_rows(dtype, d):
    """A NaN in one document's key: that document's queries are NaN, no other's; a key of -inf products counts as none; a query
    whose scores are all -inf has no keys."""
    p = Packed(dtype, d, 1, 1, (40, 40, 40), (50, 50, 50), seed=9)
    p.k[20, 0, 0] = float("nan")
    p.q[40:80, 0] = p.q[40:80, 0].abs()
    p.k[50:100, 0, :] = -float("inf")
    p.k[120, 0, :] = -float("inf")
    p.q[80:, 0] = p.q[80:, 0].abs() + 0.01
    p.forward()
    out, lse = host(p.out)[:, 0], host(p.lse)[0]
    assert np.isnan(out[:40]).all() and np.isnan(lse[:40]).all()
    assert np.all(out[40:80] == 0) and np.all(lse[40:80] == -np.inf)
    assert np.isfinite(out[80:]).all() and np.isfinite(lse[80:]).all()
    q, k, v = (host(t)[:, :1].astype(np.float64) for t in (p.q, p.k, p.v))
    ref, _, _ = train.attention(q[80:], np.delete(k[100:], 20, 0), np.delete(v[100:], 20, 0), [0, 40], [0, 49], p.scale)
    assert np.abs(out[80:] - ref[:, 0]).max() < (0.03 if dtype == "bf16" else 1e-4)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("most", [2, 4, 9, 33])
def test_attention_gradients_of_short_documents_carry_two_roundings(d, most):
    """bf16: a correctly rounded value is 2^-8 / sqrt(12) = 0.0011 to 0.0023 of itself off in the mean (0.00166 over evenly spread mantissas).  Gradients of the scores
    and results are rounded, each once: 0.00166 sqrt(2) = 0.00235; the output's own rounding must not come on top where few keys do not average it out."""
    r = np.random.default_rng(most)
    lens = [int(n) for n in r.integers(2, most + 1, 60)]
    p = Packed("bf16", d, 4, 4, lens, lens, seed=d + most).run()
    q, k, v, do = (host(t) for t in (p.q, p.k, p.v, p.dout))
    refs, _ = train.attention_grad(do, q, k, v, p.q_off, p.k_off, p.scale)
    for t, ref in zip((p.dq, p.dk, p.dv), refs):
        assert np.linalg.norm(host(t) - ref) < 0.0027 * np.linalg.norm(ref)


def test_attention_offsets_out_of_range_stay_inside(lib):
    """Offsets that descend or point past the end: taken as the nearest end, nothing outside the documents' rows is touched."""
    p = Packed("f32", 16, 1, 1, (10, 10), (10, 10))
    p.qo, p.ko = dev(np.array([-5, 8, 400], np.int32)), dev(np.array([-9, 10, 1 << 30], np.int32))
    p.q_off, p.k_off = [0, 8, 20], [0, 10, 20]
    p.run()


def test_attention_gradients_against_differences():
    """Slopes of sum(out w) in fp32: the second-order term of a step of h = 2^-6 along unit-sized directions is below 1e-3 of the sum of magnitudes."""
    p = Packed("f32", 32, 4, 2, (33, 65), (70, 12), seed=5)
    p.run()
    w, grads = host(p.dout).astype(np.float64), [host(t).astype(np.float64) for t in (p.dq, p.dk, p.dv)]
    r, h = np.random.default_rng(6), 2.0 ** -6
    for t, g in zip((p.q, p.k, p.v), grads):
        d = r.standard_normal(tuple(t.shape)).astype(np.float32)
        d /= np.sqrt(t.shape[0] * t.shape[1])
        keep, f = t.clone(), []
        for sign in (1, -1):
            t.copy_(keep + sign * h * dev(d))
            p.forward()
            f.append((host(p.out).astype(np.float64) * w).sum())
        t.copy_(keep)
        assert abs((f[0] - f[1]) / (2 * h) - (g * d).sum()) < 1e-3 * np.abs(g * d).sum()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_attention_equal_bits_on_a_side_stream_and_in_a_graph(dtype, d):
    p = Packed(dtype, d, 4, 2, (200, 77, 300), (200, 90, 300), seed=7)
    p.run()
    want = [host(t).copy() for t in (p.out, p.lse, p.dq, p.dk, p.dv)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def both():
        p.forward()
        p.backward()

    with torch.cuda.stream(side):
        both()
    side.synchronize()
    assert all(np.array_equal(host(t), x) for t, x in zip((p.out, p.lse, p.dq, p.dk, p.dv), want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for _ in range(3):
        for t in (p.out, p.lse, p.dq, p.dk, p.dv):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(host(t), x) for t, x in zip((p.out, p.lse, p.dq, p.dk, p.dv), want))


# ----------------------------------------------------------------------------------------------------------- LayerNorm
def norm_case(dtype, H, lens, groups, seed=0, front=0, back=0, residual=True, offset=0.5):
    r = np.random.default_rng(seed)
    off = front + np.cumsum((0,) + tuple(lens))
    R, G, A = int(off[-1]) + back, max(list(groups) + [0]) + 2, 3 * H + 4
    f = lambda *s: r.standard_normal(s).astype(np.float32)
    x, mods, dout, res = f(R, H) * 1.5 + offset, f(G, A), dev(f(R, H), TYPES[dtype]), f(R, H)
    shift_off, scale_off = H + 4, 0
    out, mean, rstd = torch.full((R, H), 7.0, device=DEV).to(TYPES[dtype]), torch.full((R,), 7.0, device=DEV), torch.full((R,), 7.0, device=DEV)
    dx, dmods = torch.full((R, H), 7.0, device=DEV), torch.full((G, A), 7.0, device=DEV)
    row_off, group = dev(off.astype(np.int32)), dev(np.array(groups, np.int32))
    xd, md, rd = dev(x), dev(mods), dev(res) if residual else None
    br.layer_norm_forward(xd, md, shift_off, scale_off, row_off, group, out, mean, rstd)
    ws = bytes_buffer(br.layer_norm_workspace_bytes(xd, dout, md, shift_off, scale_off, row_off, group))
    br.layer_norm_backward(dout, xd, mean, rstd, md, shift_off, scale_off, row_off, group, rd, dx, dmods, ws)

    ref, mu, rs = train.layer_norm(x, mods, shift_off, scale_off, off, groups)
    live = ~np.isnan(ref[:, 0])
    # fp32 sums of H terms, at most H / 256 + 12 of them one after the other, in the mean and the variance: c; bf16 rounds the result once,
    # by half a unit of its eighth bit: 2^-8 of the result's size at most
    c, low = (H / 256 + 16) * 2.0 ** -24, 2.0 ** -8 if dtype == "bf16" else 0.0
    o, m, s = host(out), host(mean), host(rstd)
    size = np.abs(x).max(1)
    assert np.all(np.abs(m - mu)[live] <= c * size[live]) and np.all(np.abs(s / rs - 1)[live] <= 4 * c * (size * rs)[live] ** 2 + 4 * c)
    y = np.abs(ref) + (np.abs(x - mu[:, None]) + size[:, None]) * rs[:, None] * 3
    assert np.all(np.abs(o - ref)[live] <= ((low * np.abs(ref) + 8 * c * y * (1 + (size * rs)[:, None]) * (1 + np.abs(mods[:, scale_off:scale_off + H]).max())))[live])
    assert np.all(o[~live] == 7.0) and np.all(m[~live] == 7.0)
    dh = host(dout)
    rdx, rsh, rsc = train.layer_norm_grad(dh, x, np.where(live, m, 0), np.where(live, s, 0), mods, shift_off, scale_off, off, groups, res if residual else None)
    g = np.abs(dh) * (1 + np.abs(mods).max())
    yy = np.abs((x - m[:, None]) * s[:, None])
    w = np.abs(res if residual else 0) + s[:, None] * (g + g.mean(1, keepdims=True) + yy * (g * yy).mean(1, keepdims=True))
    d = host(dx)
    assert np.all(np.abs(d - rdx)[live] <= 8 * c * w[live]), np.max((np.abs(d - rdx) / w)[live])
    assert np.all(d[~live] == 7.0)
    # column sums: at most R terms one after the other
    dm, n = host(dmods), (R / 16 + 48) * 2.0 ** -24
    absolute = np.zeros((2, G, H))
    for (a, b), k in zip(train.spans(off, R), groups):
        if 0 <= k < G:
            absolute[0, k] += np.abs(dh[a:b]).sum(0)
            absolute[1, k] += (np.abs(dh[a:b]) * (yy[a:b] + 1)).sum(0)
    assert np.all(np.abs(dm[:, shift_off:shift_off + H] - rsh) <= n * absolute[0] + 1e-30)
    assert np.all(np.abs(dm[:, scale_off:scale_off + H] - rsc) <= n * absolute[1] + 1e-30)
    assert np.all(dm[:, H:shift_off] == 7.0) and np.all(dm[:, shift_off + H:] == 7.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H", [4, 64, 252, 256, 320, 768, 1024, 1152, 1536, 2048, 2052, 3000, 4096, 6000, 16384])
def test_layer_norm_of_every_width(dtype, H):
    norm_case(dtype, H, (3, 0, 17, 1), (1, 0, 0, 2), seed=H, front=1, back=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_norm_many_documents_and_rows(dtype):
    norm_case(dtype, 128, tuple(int(n) for n in np.random.default_rng(1).integers(0, 60, 150)), [int(g) for g in np.random.default_rng(2).integers(0, 9, 150)], residual=False)
    norm_case(dtype, 512, (4100, 1, 900), (0, 1, 0), seed=3)
    norm_case(dtype, 64, (1,), (0,), seed=4)
    norm_case(dtype, 64, (0,), (0,), seed=4, back=3)


def test_layer_norm_leaves_documents_of_no_group_alone():
    norm_case("f32", 64, (5, 6, 7), (0, -1, 1), seed=5)


def test_layer_norm_of_rows_far_from_zero():
    """Rows around 1000 with a spread of 1.5: the variance is taken around the mean."""
    norm_case("f32", 512, (20,), (0,), seed=6, offset=1000.0)


def test_layer_norm_in_place_gradient_and_equal_bits():
    r = np.random.default_rng(7)
    x, res = dev(r.standard_normal((300, 768)).astype(np.float32)), dev(r.standard_normal((300, 768)).astype(np.float32))
    mods, dout = dev(r.standard_normal((2, 1536)).astype(np.float32)), dev(r.standard_normal((300, 768)).astype(np.float32), torch.bfloat16)
    off, group = dev(np.array([0, 100, 300], np.int32)), dev(np.array([1, 0], np.int32))
    out, mean, rstd = torch.empty_like(dout), torch.empty(300, device=DEV), torch.empty(300, device=DEV)
    br.layer_norm_forward(x, mods, 0, 768, off, group, out, mean, rstd)
    ws = bytes_buffer(br.layer_norm_workspace_bytes(x, dout, mods, 0, 768, off, group))
    got = []
    for place in (False, True, True):
        a, dm = res.clone(), torch.zeros_like(mods)
        dx = a if place else torch.empty_like(a)
        br.layer_norm_backward(dout, x, mean, rstd, mods, 0, 768, off, group, a, dx, dm, ws)
        got.append((host(dx), host(dm)))
    for d, m in got[1:]:
        assert np.array_equal(d, got[0][0]) and np.array_equal(m, got[0][1])


# ----------------------------------------------------------------------------------------------------------- objective
def objective_case(T, splits, K, trees, D, keep, mean, clip, ode=(), seed=0, n_total=0, moved=3e-4):
    r = np.random.default_rng(seed)
    t = br.Tree(T, splits, K, n_tree=trees)
    sched = synth.schedule(T, 3.0, logp_mean=mean, ode_steps=ode)
    nodes = trees * t.n_nodes
    ids = [n for n in range(nodes) if n % t.n_nodes and r.random() < keep] or [1]
    parent, first, coef = br.edge_rows(t, sched, D, ids)
    E, R = len(ids), len(parent)
    assert first[0] == 0 and first[-1] == E and np.all(np.diff(first) > 0) and np.all(np.diff(parent) > 0)
    z, v = r.standard_normal((nodes, D)).astype(np.float32), r.standard_normal((R, D)).astype(np.float32)
    for k in range(R):
        for e in range(first[k], first[k + 1]):
            assert ids[e] // t.n_nodes == parent[k] // t.n_nodes and t.parent[ids[e] % t.n_nodes] == parent[k] % t.n_nodes
            h = coef[k, 2] * (D if mean else 1)
            z[ids[e]] = coef[k, 0] * z[parent[k]] + coef[k, 1] * v[k] + (np.sqrt(0.5 / h) if h else 0.3) * r.standard_normal(D)
    _, logp, _, _ = train.objective_grad(z, v, ids, parent, first, coef, np.zeros(nodes), np.zeros(nodes), clip, E)
    move = r.standard_normal(E) * moved
    move = np.where(np.abs(np.abs(move) - clip) < 0.05 * clip, 1.2 * move, move)  # none on the clip's border
    old, adv = np.zeros(nodes, np.float32), r.standard_normal(nodes).astype(np.float32)
    old[ids] = logp - move
    i32 = lambda a: dev(np.asarray(a, np.int32))
    tables = (i32(ids), i32(parent), i32(first), dev(coef))
    zd, vd = dev(z), dev(v)
    J, new, grad, clipped = torch.empty(1, device=DEV), torch.empty(E, device=DEV), torch.full((R, D), 7.0, device=DEV), torch.full((E,), 7, dtype=torch.uint8, device=DEV)
    ws = bytes_buffer(br.grpo_backward_workspace_bytes(zd, vd, *tables))
    br.grpo_backward(zd, vd, *tables, dev(old), dev(adv), clip, J, new, grad, ws, clipped=clipped, n_total=n_total)
    n = n_total or E
    rJ, rlogp, rgrad, rclip = train.objective_grad(z, v, ids, parent, first, coef, old, adv, float(np.float32(clip)), n)
    # a difference carries the roundings of mu and of itself, 2^-22 of z's size of about 4; the sum of squares 2^-22 of itself
    size = np.array([coef[k, 2] for k in range(R) for _ in range(first[k], first[k + 1])]) * D * 64 * 2.0 ** -22
    err = size + 2.0 ** -22 * (1 + np.abs(rlogp))
    assert np.all(np.abs(host(new) - rlogp) <= err), np.max(np.abs(host(new) - rlogp) / err)
    return dict(J=float(host(J)[0]), rJ=rJ, clipped=host(clipped).astype(bool), rclip=rclip, grad=host(grad), rgrad=rgrad, adv=adv[ids], n=n, coef=coef, old=old, advn=adv, ids=ids,
                new=new, tables=tables, zd=zd, vd=vd, ws=ws, clip=clip, E=E, R=R, z=z, v=v, first=first, parent=parent)


@pytest.mark.parametrize("T,splits,K,trees,D,keep", [(4, (1,), 2, 1, 4, 1.0), (8, (2, 4, 6), 2, 1, 256, 0.5), (6, (0, 1, 2, 3), 3, 2, 1028, 0.7), (5, (), 1, 3, 20004, 1.0),
                                                   (3, (0,), 7, 1, 4096, 0.9), (12, (3, 6, 9), 2, 3, 65536, 0.4), (1, (), 1, 1, 64, 1.0)])
def test_objective_and_its_gradient(T, splits, K, trees, D, keep):
    c = objective_case(T, splits, K, trees, D, keep, True, 1e-4, seed=D)
    assert np.array_equal(c["clipped"], c["rclip"])
    assert abs(c["J"] - c["rJ"]) <= 2.0 ** -20 * np.abs(c["adv"]).sum() / c["n"] * 8
    w = np.zeros((c["R"], 1))
    for k in range(c["R"]):
        w[k] = np.abs(c["adv"][c["first"][k]:c["first"][k + 1]]).sum() / c["n"] * 2 * c["coef"][k, 2] * abs(c["coef"][k, 1])
    assert np.all(np.abs(c["grad"] - c["rgrad"]) <= w * 64 * 2.0 ** -22 + 1e-3 * 2.0 ** -10 * np.abs(c["rgrad"]))
    # the value is what the library's objective gives for the same log-densities
    J = torch.empty(1, device=DEV)
    br.grpo_objective(c["new"], dev(c["old"]), dev(c["advn"]), c["tables"][0], c["E"], c["clip"], J)
    assert abs(float(host(J)[0]) - c["J"]) <= 2.0 ** -20 * np.abs(c["adv"]).sum() / c["n"] * 8


def test_objective_sums_steps_without_noise_and_another_divisor():
    """Log-densities that are sums, steps without noise (no density, no gradient), a mean over more edges than the call has."""
    c = objective_case(6, (1, 3), 2, 2, 64, 0.8, False, 0.2, ode=(0, 4), seed=3, n_total=100, moved=0.3)
    assert np.array_equal(c["clipped"], c["rclip"])
    assert abs(c["J"] - c["rJ"]) <= 1e-3 * np.abs(c["adv"]).sum() / 100
    assert np.abs(c["grad"] - c["rgrad"]).max() <= 1e-3 * np.abs(c["rgrad"]).max()
    still = c["coef"][:, 2] == 0
    assert still.any() and np.all(c["grad"][still] == 0) and np.all(host(c["new"])[np.repeat(still, np.diff(c["first"]))] == 0)


def test_objective_gradient_against_differences():
    """Slope of J along a direction, from the kernel's own values: J is within 2^-22 of the terms' size, the step moves it by far more."""
    c = objective_case(8, (2, 4), 2, 2, 128, 0.9, True, 0.3, seed=5, moved=0.02)
    r = np.random.default_rng(6)
    d = r.standard_normal(c["v"].shape).astype(np.float32)
    h, f = 2.0 ** -6, []
    for sign in (1, -1):
        J, new, grad = torch.empty(1, device=DEV), torch.empty(c["E"], device=DEV), torch.empty_like(c["vd"])
        br.grpo_backward(c["zd"], dev(c["v"] + sign * h * d), *c["tables"], dev(c["old"]), dev(c["advn"]), c["clip"], J, new, grad, c["ws"])
        f.append(float(host(J)[0]))
    got, want = -(f[0] - f[1]) / (2 * h), (c["grad"].astype(np.float64) * d).sum()
    assert not c["clipped"].any() and abs(got - want) < 2e-2 * np.abs(c["grad"] * d).sum() / np.sqrt(c["grad"].size) + 2.0 ** -22 / h * 4


def test_objective_without_edges_and_equal_bits_in_a_graph():
    c = objective_case(8, (2,), 3, 2, 5000, 0.6, True, 1e-4, seed=9)
    J, new, grad = torch.empty(1, device=DEV), torch.empty(c["E"], device=DEV), torch.empty_like(c["vd"])
    old, adv = dev(c["old"]), dev(c["advn"])
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        br.grpo_backward(c["zd"], c["vd"], *c["tables"], old, adv, c["clip"], J, new, grad, c["ws"])
    for _ in range(3):
        grad.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(host(grad), c["grad"]) and float(host(J)[0]) == c["J"]
    e = [t[:0] for t in c["tables"]]
    br.grpo_backward(c["zd"], c["vd"][:0], e[0], e[1], c["tables"][2][:1], c["tables"][3][:0], old, adv, 0.1, J, new[:0], grad[:0], c["ws"])
    assert float(host(J)[0]) == 0.0


# --------------------------------------------------------------------------------------------------------------- AdamW
def adamw_case(sizes, bits, grads, copies, steps=3, shift=0, seed=0, scale=None, decay=0.05, eps=1e-8):
    """Tensors that begin `shift` elements into a buffer, against the oracle in fp32 with one rounding an operation: equal bits."""
    r = np.random.default_rng(seed)
    part = lambda t, n: torch.cat([torch.zeros(shift, dtype=t.dtype, device=DEV), t])[shift:shift + n]
    f = lambda n, s: (r.standard_normal(n) * s).astype(np.float32)
    P, G = [f(n, 0.02) for n in sizes], [f(n, 1e-3) for n in sizes]
    gt = [part(dev(g, TYPES[grads]), n) for g, n in zip(G, sizes)]
    G = [host(g).astype(np.float32) for g in gt]
    pt = [part(dev(p), n) for p, n in zip(P, sizes)]
    M, V = [f(n, 3e-4) for n in sizes], [np.abs(f(n, 1e-6)) for n in sizes]
    if bits == 8:
        M, V = [train.encode(m, 3, np.zeros(len(m)), True) for m in M], [train.encode(np.sqrt(v), 4, np.zeros(len(v)), False) for v in V]
        mt, vt = [part(dev(m[0]), n) for m, n in zip(M, sizes)], [part(dev(v[0]), n) for v, n in zip(V, sizes)]
        ms, vs = [dev(m[1]) for m in M], [dev(v[1]) for v in V]
    else:
        mt, vt, ms, vs = [part(dev(m), n) for m, n in zip(M, sizes)], [part(dev(v), n) for v, n in zip(V, sizes)], None, None
    ct = [part(torch.zeros(n, dtype=torch.bfloat16, device=DEV), n) if i % 2 == 0 else None for i, n in enumerate(sizes)] if copies else None
    opt = br.AdamW(pt, gt, mt, vt, ms, vs, ct, weight_decay=decay, lr=1e-3, betas=(0.9, 0.99), eps=eps, seed=77, step=4)
    st = dev(np.array([scale], np.float32)) if scale else None
    for k in range(steps):
        opt.step(grad_scale=st)
        for i, n in enumerate(sizes):
            m, v = M[i], V[i]
            if bits == 8:
                root = train.decode(*v, 4, False)
                m, v = train.decode(*m, 3, True), root * root
            g = G[i] * np.float32(scale) if scale else G[i]
            P[i], m, v, root = train.adamw(P[i], g, m, v, 5 + k, 1e-3, 0.9, 0.99, eps, decay[i] if isinstance(decay, list) else decay, np.float32)
            if bits == 8:
                w = train.adamw_words(77, i, 5 + k, n)
                M[i], V[i] = train.encode(m, 3, w & 0xFFFF, True), train.encode(root, 4, w >> 16, False)
            else:
                M[i], V[i] = m, v
    for i, n in enumerate(sizes):
        assert np.array_equal(host(pt[i]), P[i]), (i, n, np.abs(host(pt[i]) - P[i]).max())
        if bits == 8:
            assert np.array_equal(host(mt[i]), M[i][0]) and np.array_equal(host(vt[i]), V[i][0]), (i, n)
            assert np.array_equal(host(ms[i]), M[i][1]) and np.array_equal(host(vs[i]), V[i][1]), (i, n)
        else:
            assert np.array_equal(host(mt[i]), M[i]) and np.array_equal(host(vt[i]), V[i]), (i, n)
        if ct and ct[i] is not None:
            assert np.array_equal(host(ct[i]), synth.from_bf16_bits(synth.to_bf16_bits(P[i])))
    return opt, M, V


SIZES = [1, 3, 4, 63, 255, 256, 257, 1000, 0, 4096, 4097, 70001]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grads", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 4, 1, 3])
def test_adamw_bit_for_bit(bits, grads, shift):
    adamw_case(SIZES, bits, grads, True, shift=shift, seed=shift)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_more_tensors_than_a_launch_takes_and_a_factor_of_the_gradients(bits):
    adamw_case([17 + 13 * i for i in range(131)], bits, "f32", False, steps=2, scale=0.37, decay=[0.0, 0.1, 0.01] * 43 + [0.0, 0.2])


def test_adamw_values_of_states_in_8_bits():
    opt, M, V = adamw_case(SIZES, 8, "f32", False, steps=1)
    out = [[torch.full((n + 1,), 7.0, device=DEV)[1 if odd else 0:][:n] for n in SIZES] for odd in (False, True)]
    opt.state_values(*out)
    for m, v, a, b in zip(M, V, *out):
        root = train.decode(*v, 4, False)
        assert np.array_equal(host(a), train.decode(*m, 3, True)) and np.array_equal(host(b), root * root)


def test_adamw_states_in_8_bits_follow_changes_below_half_a_code():
    """A constant gradient moves a second moment by 0.1 % a step, a code is 3 to 6 % wide: to the nearest code it would never move.  After n steps v is (1 -
    0.999^n) g^2; rounding leaves each element a random walk around it, 4096 of them together stay within 2 %."""
    n = 4096
    p, g, m, v = torch.zeros(n, device=DEV), torch.full((n,), 0.01, device=DEV), *(torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
    g[::256] = 0.02  # the block's largest
    ms, vs = torch.zeros(n // 256, device=DEV), torch.zeros(n // 256, device=DEV)
    opt = br.AdamW([p], [g], [m], [v], [ms], [vs], lr=0.0, weight_decay=0.0, seed=5)
    mv, vv = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    for _ in range(1500):
        opt.step()
    opt.state_values([mv], [vv])
    rest = np.arange(n) % 256 != 0
    assert abs(np.sqrt(host(vv)[rest]).mean() / (0.01 * np.sqrt(1 - 0.999 ** 1500)) - 1) < 0.02
    assert abs(host(mv)[rest].mean() / 0.01 - 1) < 0.02


def test_adamw_marks_blocks_that_are_not_finite_and_leaves_the_others():
    n = 1024
    for bad in (float("nan"), float("inf")):
        g, p, m, v = torch.full((n,), 0.01, device=DEV), torch.ones(n, device=DEV), *(torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
        g[300] = bad
        opt = br.AdamW([p], [g], [m], [v], [torch.zeros(4, device=DEV)], [torch.zeros(4, device=DEV)], lr=0.1, weight_decay=0.0)
        mv, vv = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        opt.step()
        opt.state_values([mv], [vv])
        hit = (np.arange(n) // 256) == 1
        for t in (host(mv), host(vv)):
            assert np.isnan(t[hit]).all() and np.isfinite(t[~hit]).all()
        assert np.isfinite(np.delete(host(p), 300)).all() and np.isnan(host(p)[300])


def test_adamw_in_a_graph_with_a_factor_that_changes():
    """A captured step: the pointers travel in the kernel's arguments, the factor is read when the step runs."""
    n = 5000
    r = np.random.default_rng(3)
    p0, g0 = r.standard_normal(n).astype(np.float32), r.standard_normal(n).astype(np.float32)
    p, g, m, v, s = dev(p0), dev(g0), torch.zeros(n, device=DEV), torch.zeros(n, device=DEV), torch.ones(1, device=DEV)
    opt = br.AdamW([p], [g], [m], [v], lr=0.01, weight_decay=0.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step(grad_scale=s)
    P, M, V = p0, np.zeros(n, np.float32), np.zeros(n, np.float32)
    for k in range(3):
        s.fill_(0.5 + k)
        graph.replay()
        torch.cuda.synchronize()
        P, M, V, _ = train.adamw(P, g0 * np.float32(0.5 + k), M, V, 1, 0.01, 0.9, 0.999, 1e-8, 0.0, np.float32)
        assert np.array_equal(host(p), P) and np.array_equal(host(m), M) and np.array_equal(host(v), V)
