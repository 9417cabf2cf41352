"""Workspaces of the training operators: never above the bounds that the header states, which callers allocate by, over small and large calls and over the performance cases."""
import ctypes as C
import importlib.util
import os
import random

import pytest

from paper_2509_06040_amd import binding as br

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = C.c_void_p(1 << 20)  # an address that nothing reads


def operators():
    spec = importlib.util.spec_from_file_location("perf_operators", os.path.join(ROOT, "perf", "operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def norm_need(dtype, rows, hidden, docs, groups=1):
    s = br.NormShape(dtype, rows, hidden, docs, groups, 2 * hidden, 0, hidden, P.value, P.value)
    need = br.load().br_layer_norm_workspace_bytes(C.byref(s))
    assert need > 0
    return need


@pytest.mark.parametrize("hidden", [4, 32, 64, 128, 192, 320, 512, 768, 1024, 1152, 1536, 2048, 3000, 4096, 16384])
def test_layer_norm_workspace_stays_within_its_bound(hidden):
    """Column sums of a tile for every 16 rows, two a document and 1024 besides."""
    r = random.Random(hidden)
    rows = sorted({0, 1, 15, 16, 17, 4095, 4096, 1 << 20, 1 << 24} | set(range(5000, 20001, 173)) | {int(2 ** r.uniform(0, 24)) for _ in range(200)})
    for n in rows:
        for docs in (0, 1, 2, 16, 48, 1000):
            assert norm_need(br.BF16, n, hidden, docs) <= 8 * max(hidden, 64) * (n // 16 + 2 * docs + 1024), (n, docs)


def test_workspaces_of_the_performance_cases_fit_what_these_allocate():
    ops, rng, seen = operators(), random.Random(5), set()
    for _ in range(4000):
        c = ops.draw(rng)
        seen.add(c["kind"])
        t = br.BF16 if c.get("dtype") == "bf16" else br.F32
        if c["kind"] == "norm":
            lens = ops._lengths(c)[0]
            assert norm_need(t, sum(lens), c["hidden"], len(lens), c["groups"]) <= 8 * c["hidden"] * (sum(lens) // 16 + 2 * len(lens) + 1024), c
        if c["kind"] == "attention":
            lq, lk = ops._lengths(c)
            nh, nkv, d = c["heads"], c["kv_heads"], c["head_dim"]
            s = br.AttnShape(t, nh, nkv, d, len(lq), sum(lq), sum(lk), 0.0, *[(nh + 2 * nkv) * d] * 3, nh * d, *[(nh + 2 * nkv) * d] * 3, P.value, P.value)
            assert br.load().br_attention_workspace_bytes(C.byref(s), int(c["way"] == "bwd")) <= 8 * nh * sum(lq) + (1 << 27), c
        if c["kind"] == "objective":
            nodes, edges, rows, _, _ = ops._tables(c)
            s = br.EdgeSet(c["D"], nodes, len(rows), len(edges), 0, 0.1, P.value, P.value, P.value, P.value)
            assert 0 < br.load().br_grpo_backward_workspace_bytes(C.byref(s)) <= 8 * (len(edges) * (c["D"] // 1024 + 2) + 1024), c
    assert {"norm", "attention", "objective"} <= seen


@pytest.mark.parametrize("groups,docs,ok", [(65535, 2046, True), (65535, 2047, False), (15360, 15360, True), (16384, 16384, False), (1, 1 << 24, True), (17, 1 << 24, False)])
def test_layer_norm_backward_refuses_groups_times_documents_that_would_take_seconds(groups, docs, ok):
    """The join reads every tile once for each group; forward has no such join."""
    s = br.NormShape(br.BF16, 1 << 20, 64, docs, groups, 128, 0, 64, P.value, P.value)
    lib = br.load()
    assert (lib.br_layer_norm_workspace_bytes(C.byref(s)) > 0) == ok
    if not ok:
        assert lib.br_layer_norm_backward(C.byref(s), P, P, P, P, P, None, P, P, P, C.c_size_t(1 << 50), None) == -3
        assert b"br_layer_norm_backward" in lib.br_last_error() and b"groups" in lib.br_last_error()
