"""Refusals and host tables of the operators of a policy update.  No kernel is launched here: every call ends at its argument checks."""
import ctypes as C
import os
import re

import numpy as np
import pytest

from oracle import tree
from paper_2509_06040_amd import binding as br
from paper_2509_06040_amd import synth

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, ODD, SIZE = C.c_void_p(1 << 20), C.c_void_p((1 << 20) + 4), C.c_size_t(1 << 40)  # addresses that nothing reads
EINVAL, ESHAPE, EWORKSPACE = -1, -3, -4


def test_library_exports_the_declared_symbols():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "branchrollout_train.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(br_[a-z0-9_]+)\s*\(", text))
    assert declared == set(br.TRAIN_EXPORTS) and all(hasattr(br.load(), n) for n in declared)


def refused(code, name, *args):
    lib = br.load()
    assert getattr(lib, name)(*args) == code, (name, lib.br_last_error())
    assert name.encode() in lib.br_last_error()


def attn(**change):
    s = br.AttnShape(br.BF16, 4, 2, 64, 3, 100, 120, 0.0, 256, 128, 128, 256, 256, 128, 128, P.value, P.value)
    for k, v in change.items():
        setattr(s, k, v)
    return s


def test_attention_refuses():
    def forward(code, s, q=P, lse=P, ws=P, room=SIZE):
        refused(code, "br_attention_forward", C.byref(s) if s else None, q, P, P, P, lse, ws, room, None)

    forward(EINVAL, None)
    for change in (dict(dtype=2), dict(n_heads=3), dict(n_kv_heads=0), dict(n_docs=-1), dict(q_tokens=-1), dict(q_off=None), dict(scale=float("nan")), dict(scale=-1.0)):
        forward(EINVAL, attn(**change))
        assert br.load().br_attention_workspace_bytes(C.byref(attn(**change)), 1) == 0
    for change in (dict(head_dim=32), dict(head_dim=96), dict(q_stride=252), dict(q_stride=248), dict(k_stride=64), dict(v_stride=1 << 40), dict(o_stride=0)):
        forward(ESHAPE, attn(**change))
    forward(ESHAPE, attn(dtype=br.F32, head_dim=8))
    forward(EINVAL, attn(), q=None)
    forward(EINVAL, attn(), lse=None)
    forward(ESHAPE, attn(), q=ODD)

    def backward(code, s, dq=P, ws=P, room=SIZE):
        refused(code, "br_attention_backward", C.byref(s), P, P, P, P, P, P, dq, P, P, ws, room, None)

    backward(ESHAPE, attn(dq_stride=128))
    backward(EINVAL, attn(), dq=None)
    backward(ESHAPE, attn(), dq=ODD)
    need = br.load().br_attention_workspace_bytes(C.byref(attn()), 1)
    assert need > 0
    backward(EWORKSPACE, attn(), ws=None)
    backward(EWORKSPACE, attn(), room=C.c_size_t(need - 1))


def norm(**change):
    s = br.NormShape(br.BF16, 100, 64, 3, 2, 384, 0, 64, P.value, P.value)
    for k, v in change.items():
        setattr(s, k, v)
    return s


def test_layer_norm_refuses():
    def forward(code, s, x=P, mean=P, rstd=P):
        refused(code, "br_layer_norm_forward", C.byref(s) if s else None, x, P, P, mean, rstd, None)

    forward(EINVAL, None)
    for change in (dict(dtype=3), dict(rows=-1), dict(n_groups=0), dict(row_off=None), dict(group=None), dict(shift_off=-4), dict(scale_off=324)):
        forward(EINVAL, norm(**change))
        assert br.load().br_layer_norm_workspace_bytes(C.byref(norm(**change))) == 0
    for change in (dict(hidden=66), dict(mods_stride=386), dict(hidden=16388, mods_stride=1 << 20), dict(n_groups=1 << 20)):
        forward(ESHAPE, norm(**change))
    forward(EINVAL, norm(), x=None)
    forward(EINVAL, norm(), mean=None)
    forward(ESHAPE, norm(), x=ODD)

    def backward(code, s, dx=P, room=SIZE):
        refused(code, "br_layer_norm_backward", C.byref(s), P, P, P, P, P, None, dx, P, P, room, None)

    backward(EINVAL, norm(scale_off=32))
    backward(EINVAL, norm(), dx=None)
    backward(EWORKSPACE, norm(), room=C.c_size_t(br.load().br_layer_norm_workspace_bytes(C.byref(norm())) - 1))


def edges(**change):
    s = br.EdgeSet(64, 50, 3, 5, 0, 0.1, P.value, P.value, P.value, P.value)
    for k, v in change.items():
        setattr(s, k, v)
    return s


def test_objective_refuses():
    def call(code, s, z=P, J=P, room=SIZE):
        refused(code, "br_grpo_backward", C.byref(s) if s else None, z, P, P, P, J, P, P, None, P, room, None)

    call(EINVAL, None)
    for change in (dict(D=0), dict(n_rows=6), dict(n_rows=0), dict(n_total=-1), dict(n_nodes=0), dict(clip_eps=-0.1), dict(clip_eps=float("inf")), dict(row_coef=None)):
        call(EINVAL, edges(**change))
        assert br.load().br_grpo_backward_workspace_bytes(C.byref(edges(**change))) == 0
    call(ESHAPE, edges(D=66))
    call(EINVAL, edges(), z=None)
    call(EINVAL, edges(), J=None)
    call(ESHAPE, edges(), z=ODD)
    call(EWORKSPACE, edges(), room=C.c_size_t(8))


def test_adamw_refuses():
    def tensor(**change):
        t = br.AdamwTensor(P.value, P.value, P.value, P.value, P.value, P.value, P.value, 10, 0.1)
        for k, v in change.items():
            setattr(t, k, v)
        return t

    def call(code, t=None, n=1, **change):
        c = br.AdamwCfg(1e-3, 0.9, 0.999, 1e-8, 1, 0, br.F32, 8, None)
        for k, v in change.items():
            setattr(c, k, v)
        refused(code, "br_adamw_step", C.byref(c), C.byref(t) if t else None, C.c_int32(n), None)

    call(EINVAL)
    call(EINVAL, tensor(), n=-1)
    for change in (dict(grad_dtype=2), dict(state_bits=16), dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(lr=float("nan"))):
        call(EINVAL, tensor(), **change)
    for change in (dict(n=-1), dict(param=None), dict(grad=None), dict(m=None), dict(v_scale=None), dict(weight_decay=float("inf"))):
        call(EINVAL, tensor(**change))
    for change in (dict(n=1 << 35), dict(param=P.value + 2), dict(grad=P.value + 2), dict(copy=P.value + 1)):
        call(ESHAPE, tensor(**change))
    call(ESHAPE, tensor(m=P.value + 2), state_bits=32)
    refused(EINVAL, "br_adamw_state_values", C.byref(tensor()), C.c_int32(1), None, P, None)


def test_edge_rows_are_the_distinct_parents_with_their_steps():
    t, o = br.Tree(6, (1, 3), 3, n_tree=2), tree.tree_build(6, (1, 3), 3)
    sched = synth.schedule(6, 3.0, logp_mean=True, ode_steps=(2,))
    r = np.random.default_rng(0)
    ids = [n for n in range(2 * t.n_nodes) if n % t.n_nodes and r.random() < 0.6]
    parent, first, coef = br.edge_rows(t, sched, 100, ids)
    of = [e // t.n_nodes * t.n_nodes + o["parent"][e % t.n_nodes] for e in ids]
    assert list(parent) == sorted(set(of)) and [parent[k] for k in range(len(parent)) for _ in range(first[k], first[k + 1])] == of
    for k, p in enumerate(parent):
        i = o["depth"][p % t.n_nodes]
        s, a, b = float(sched["sigma"][i]), float(sched["t"][i]), float(sched["t"][i + 1])
        g = (a - b) * s * s / (2 * a)
        want = (1 - g, -(a - b) - g * (1 - a), 0.5 / (s * s * (a - b)) / 100 if s else 0, -0.5 * np.log(s * s * (a - b) * 2 * np.pi) if s else 0)
        assert np.allclose(coef[k], want, rtol=1e-6, atol=1e-12)


def test_edge_rows_refuse():
    t, sched = br.Tree(4, (1,), 2), synth.schedule(4, 3.0)
    for ids in ([0], [2, 2], [3, 2], [-1], [t.n_nodes]):
        with pytest.raises(br.BranchRolloutError) as e:
            br.edge_rows(t, sched, 8, ids)
        assert e.value.code == EINVAL
    with pytest.raises(br.BranchRolloutError):
        br.edge_rows(t, synth.schedule(5, 3.0), 8, [1])
    assert [len(x) for x in br.edge_rows(t, sched, 8, [])] == [0, 1, 0]


def test_packed_shapes_are_laid_out_as_the_structures():
    for packed, fields in ((br._ATTN_SHAPE, br.AttnShape), (br._NORM_SHAPE, br.NormShape), (br._EDGE_SET, br.EdgeSet)):
        values = [k + 1 for k in range(len(fields._fields_))]
        assert packed.size == C.sizeof(fields) and [getattr(fields.from_buffer_copy(packed.pack(*values)), n) for n, _ in fields._fields_] == values
