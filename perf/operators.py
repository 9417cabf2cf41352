"""Performance cases of the operators that train the policy: what follows a rollout, once its kept edges and advantages are known.

A case is a dict of plain values.  `kind` names the operator:
  attention  softmax(Q K^T scale) V over documents of ragged lengths packed along the tokens, heads of queries that may share heads of
             keys and values; `way` fwd: output and log-sum-exp, bwd: the gradients of queries, keys and values
  norm       LayerNorm modulated by the shift and scale of each document's condition; `way` fwd: output, mean and 1/std of the rows,
             bwd: gradient of the rows (with the gradient that the residual stream carries past the norm) and of the conditions' vectors
  objective  the clipped objective over kept edges and its gradient with respect to the velocities at the edges' parents
  adamw      one AdamW step over all tensors of a network, states in 32 bits or in 8, with the bf16 copies that the network reads
`own` False computes the operators in plain torch operations in 32 bits, True by the library's entry points.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------------------- cases
def _attention(way, dtype, heads, kv_heads, head_dim, docs, image, prompt, cross=False, mix=1):
    return dict(kind="attention", way=way, dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, docs=docs, image=image,
                prompt=prompt, cross=cross, mix=mix)


def _norm(way, dtype, hidden, docs, image, prompt, groups, mix=1):
    return dict(kind="norm", way=way, dtype=dtype, hidden=hidden, docs=docs, image=image, prompt=prompt, groups=groups, mix=mix)


def _objective(T, splits, K, trees, D, kept, mix=1):
    return dict(kind="objective", T=T, splits=",".join(map(str, splits)), K=K, trees=trees, D=D, kept=kept, mix=mix)


def _adamw(blocks, hidden, tokens, patch, bits, grads, copies, align=256, mix=1):
    return dict(kind="adamw", blocks=blocks, hidden=hidden, tokens=tokens, patch=patch, bits=bits, grads=grads, copies=copies,
                align=align, mix=mix)


def listed():
    return [
        # the image network (16 heads of 64, 1024 latent tokens), a frontier of 16 samples whose prompts have 1 to 77 tokens
        dict(_attention("fwd", "bf16", 16, 16, 64, 16, 1024, 77), name="attention forward image"),
        # the same in the update, 8 samples a micro-batch
        dict(_attention("bwd", "bf16", 16, 16, 64, 8, 1024, 77), name="attention backward image"),
        # 4096 latent tokens and prompts up to 512, 12 heads of 128: the longest sequence whose plain form fits the card
        dict(_attention("bwd", "bf16", 12, 12, 128, 2, 4096, 512), name="attention backward large"),
        # latents that look at their prompts, some of them empty (the unconditional samples), fp32, heads of 16 of the fp32 reference network
        dict(_attention("fwd", "f32", 4, 4, 16, 8, 16, 8, cross=True), name="attention forward tiny"),
        # fp32, eight heads of queries on two of keys and values, documents from a few to 400 tokens
        dict(_attention("bwd", "f32", 8, 2, 64, 6, 4, 400), name="attention backward shared"),
        # the image network's frontier of 16 samples, four conditions
        dict(_norm("fwd", "bf16", 1024, 16, 1024, 77, 4), name="norm forward image"),
        # one video sample and its prompt: 33 000 rows of 1536
        dict(_norm("bwd", "bf16", 1536, 1, 32760, 512, 1), name="norm backward video"),
        # the fp32 reference tree: every call is a few kilobytes
        dict(_objective(8, (2, 4, 6), 2, 1, 256, 0.5), name="objective tiny"),
        # the image workload: four trees of 16 leaves, latents of 65 536 values, half of the edges kept
        dict(_objective(20, (4, 8, 12, 16), 2, 4, 65536, 0.5), name="objective image"),
        # the fp32 reference network: 23 small tensors, launch cost
        dict(_adamw(2, 64, 16, 16, 32, "f32", False), name="adamw tiny"),
        # the image network's 240 M parameters, states in 32 bits, gradients in bf16
        dict(_adamw(12, 1024, 1024, 64, 32, "bf16", True), name="adamw image 32 bit"),
        # the same with states in 8 bits
        dict(_adamw(12, 1024, 1024, 64, 8, "bf16", True), name="adamw image 8 bit"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("attention", "attention", "norm", "objective", "adamw"))
    mix = rng.randrange(1 << 30)
    way, dtype = rng.choice(("fwd", "bwd")), rng.choice(("bf16", "f32"))
    if kind == "attention":
        head_dim = rng.choice((64, 128) if dtype == "bf16" else (16, 32, 64, 128))
        kv_heads, share = rng.choice((1, 2, 3, 4, 6, 8)), rng.choice((1, 1, 1, 2, 4))
        heads = kv_heads * share
        docs = _log(rng, 1, 24)
        most = min(2048 if dtype == "bf16" else 1024, int(math.sqrt(2.4e8 / (docs * heads))))
        tokens = _log(rng, 4, most)
        prompt = max(1, int(tokens * rng.uniform(0.05, 0.9)))
        return _attention(way, dtype, heads, kv_heads, head_dim, docs, tokens - prompt, prompt, cross=rng.random() < 0.3, mix=mix)
    if kind == "norm":
        hidden = rng.choice((64, 128, 192, 320, 512, 768, 1024, 1152, 1536, 2048))
        docs = _log(rng, 1, 48)
        tokens = _log(rng, 1, max(1, min(4096, 40_000_000 // (hidden * docs))))
        prompt = max(1, int(tokens * rng.uniform(0.05, 1.0)))
        return _norm(way, dtype, hidden, docs, tokens - prompt, prompt, rng.randint(1, docs), mix=mix)
    if kind == "objective":
        T, K = rng.randint(4, 20), rng.choice((1, 2, 3))
        splits = sorted(rng.sample(range(T), rng.randint(0, min(3, T))))
        trees, D = rng.randint(1, 4), 4 * _log(rng, 16, 50_000)
        if trees * T * K ** len(splits) * D > 30_000_000:
            trees, D = 1, D // 16 // 4 * 4 + 4
        return _objective(T, splits, K, trees, D, round(rng.uniform(0.2, 1.0), 2), mix=mix)
    bits, grads = rng.choice((8, 32)), rng.choice(("f32", "bf16"))
    return _adamw(rng.randint(1, 8), 8 * _log(rng, 4, 96), rng.randint(4, 500), 4 * rng.randint(1, 32), bits, grads, copies=rng.random() < 0.7,
                  align=rng.choice((256, 512) if bits == 8 else (1, 256)), mix=mix)


# ------------------------------------------------------------------------------------------------- shapes out of a case
def _lengths(c):
    """(tokens of queries, tokens of keys) of each document.  Joint sequences: latent tokens and 1 .. prompt tokens of a prompt; cross: latent
    tokens against prompts and an end mark, one document in four or so without any."""
    rng = random.Random(c["mix"])
    p = [rng.randint(1, c["prompt"]) for _ in range(c["docs"])]
    if not c.get("cross"):
        n = [c["image"] + x for x in p]
        return n, n
    return [c["image"] for _ in p], [0 if i and rng.random() < 0.25 else x + 1 for i, x in enumerate(p)]


def _tree(c):
    """(parent, step) of every node but the roots, in level order over all trees; ids of the kept edges (their children), ascending."""
    splits = {int(s) for s in c["splits"].split(",") if s}
    parent, step, at, level = [-1], [-1], [0], 1
    for i in range(c["T"]):
        below = []
        for p in at:
            for _ in range(c["K"] if i in splits else 1):
                below.append(level)
                parent.append(p)
                step.append(i)
                level += 1
        at = below
    rng = random.Random(c["mix"])
    n, edges = len(parent), []
    for t in range(c["trees"]):
        edges += [t * n + k for k in range(1, n) if rng.random() < c["kept"]]
    edges = edges or [1]
    return n, parent, step, edges


def _tables(c):
    """What a program keeps of its kept edges: rows = their distinct parents in ascending order, each with its first edge, its node and its
    coefficients: mean of the step a_z z + a_v v, log-density c0 - h |z_child - mean|^2 (divided by the latent's size)."""
    n, parent, step, edges = _tree(c)
    T, D = c["T"], c["D"]
    u = 1.0 - np.arange(T + 1) / T
    t = (3.0 * u / (1.0 + 2.0 * u)).astype(np.float32).astype(np.float64)
    row_parent, row_first, coef = [], [], []
    for e, child in enumerate(edges):
        p = child // n * n + parent[child % n]
        if not row_parent or row_parent[-1] != p:
            i = step[child % n]
            h, s = t[i] - t[i + 1], float(np.float32(0.3))
            g = h * s * s / (2.0 * t[i])
            var = s * s * h
            row_parent.append(p)
            row_first.append(e)
            coef.append((1.0 - g, -h - g * (1.0 - t[i]), 1.0 / (2.0 * var * D), -0.5 * math.log(var) - 0.5 * math.log(2.0 * math.pi)))
    return n * c["trees"], edges, row_parent, row_first + [len(edges)], coef


def _parameters(c):
    """(elements, whether a matrix) of a network's tensors, those of the blocks stacked."""
    H, N, pd = c["hidden"], c["blocks"], c["patch"]
    A = N * 6 * H + 2 * H
    return [(H * pd, True), (H, False), (c["tokens"] * H, False), (H * H, True), (H, False), (H * 256, True), (H, False), (H * H, True),
            (H, False), (H * H, True), (H, False), (A * H, True), (A, False), (N * 3 * H * H, True), (N * 3 * H, False), (N * H * H, True),
            (N * H, False), (N * 4 * H * H, True), (N * 4 * H, False), (N * 4 * H * H, True), (N * H, False), (pd * H, True), (pd, False)]


def _places(c):
    """Where each tensor begins in the program's one buffer of a kind, and the buffer's size."""
    at, size = [], 0
    for n, _ in _parameters(c):
        at.append(size)
        size += -(-n // c["align"]) * c["align"]
    return at, size


def work(case):
    c = case
    if c["kind"] == "attention":
        q, k = _lengths(c)
        b = 2 if c["dtype"] == "bf16" else 4
        nq, nk = sum(q) * c["heads"] * c["head_dim"], sum(k) * c["kv_heads"] * c["head_dim"]
        unit = 2.0 * sum(x * y for x, y in zip(q, k)) * c["heads"] * c["head_dim"]
        if c["way"] == "fwd":
            return {"bytes": b * (2 * nq + 2 * nk) + 4 * sum(q) * c["heads"], "flops": 2 * unit}
        return {"bytes": b * (3 * nq + 4 * nk) + 4 * sum(q) * c["heads"], "flops": 5 * unit}
    if c["kind"] == "norm":
        R, b = sum(_lengths(c)[0]), 2 if c["dtype"] == "bf16" else 4
        n, v = R * c["hidden"], c["groups"] * c["hidden"]
        if c["way"] == "fwd":
            return {"bytes": n * (4 + b) + 8 * v + 8 * R, "flops": 8 * n}
        return {"bytes": n * (4 + b + 4 + 4) + 12 * v + 8 * R, "flops": 16 * n}
    if c["kind"] == "objective":
        _, edges, rows, _, _ = _tables(c)
        nodes = len(set(edges) | set(rows))
        return {"bytes": 4.0 * c["D"] * (nodes + 2 * len(rows)), "flops": 10.0 * c["D"] * len(edges)}
    n, g = sum(x for x, _ in _parameters(c)), 2 if c["grads"] == "bf16" else 4
    m = sum(x for x, is_matrix in _parameters(c) if is_matrix) if c["copies"] else 0
    state = 16 * n if c["bits"] == 32 else 4 * n + 16 * (n // 256) + 8 * n  # 8 bits: codes and scales both ways, and the values read out of them
    return {"bytes": n * (8 + g) + 2 * m + state, "flops": 15.0 * n}


# -------------------------------------------------------------------------------------------------------------- inputs
def _ints(v):
    return torch.tensor(v, dtype=torch.int32).to(DEV)


def _offsets(n):
    return _ints(np.concatenate([[0], np.cumsum(n)]).tolist())


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device=DEV)  # noqa: E731
    return {"attention": _prepare_attention, "norm": _prepare_norm, "objective": _prepare_objective, "adamw": _prepare_adamw}[case["kind"]](case, g, normal)


def _prepare_attention(c, g, normal):
    lq, lk = _lengths(c)
    Tq, Tk, T = sum(lq), sum(lk), DTYPES[c["dtype"]]
    NH, NKV, d = c["heads"], c["kv_heads"], c["head_dim"]
    s = dict(case=c, q_off=_offsets(lq), k_off=_offsets(lk), most_q=max(lq), most_k=max(max(lk), 1))
    for name in ("", "d"):  # the projections' output, and its gradient: queries, keys and values of a token side by side
        if c["cross"]:
            q, kv = normal(Tq, NH, d).to(T), normal(Tk, 2 * NKV, d).to(T)
        else:
            q = normal(Tq, NH + 2 * NKV, d).to(T)
            q, kv = q[:, :NH], q[:, NH:]
        s[name + "q"], s[name + "k"], s[name + "v"] = q, kv[:, :NKV], kv[:, NKV:]
    s["out"], s["lse"] = torch.empty(Tq, NH, d, dtype=T, device=DEV), torch.empty(NH, Tq, device=DEV)
    if c["way"] == "bwd":
        s["dout"] = normal(Tq, NH, d).to(T)
        s["out"], s["lse"] = _plain_attention_forward(s)
    s["work"] = torch.empty(8 * NH * Tq + (1 << 27), dtype=torch.uint8, device=DEV)
    return s


def _prepare_norm(c, g, normal):
    lens, H, G, T = _lengths(c)[0], c["hidden"], c["groups"], DTYPES[c["dtype"]]
    R, A = sum(lens), 8 * H  # a block's six vectors and the last layer's two
    rng = random.Random(c["mix"] + 1)
    s = dict(case=c, row_off=_offsets(lens), group=_ints([rng.randrange(G) for _ in lens]), shift_off=3 * H, scale_off=4 * H,
             x=normal(R, H) * 2 + normal(R, 1) * 0.5, mods=normal(G, A) * 0.3,
             out=torch.empty(R, H, dtype=T, device=DEV), mean=torch.empty(R, device=DEV), rstd=torch.empty(R, device=DEV))
    if c["way"] == "bwd":
        s["dout"], s["residual"] = normal(R, H).to(T), normal(R, H)
        s["mean"] = s["x"].mean(1)
        s["rstd"] = torch.rsqrt(((s["x"] - s["mean"][:, None]) ** 2).mean(1) + 1e-6)
        s["dx"], s["dmods"] = torch.empty(R, H, device=DEV), torch.zeros(G, A, device=DEV)
        s["work"] = torch.empty(8 * H * (R // 16 + 2 * len(lens) + 1024), dtype=torch.uint8, device=DEV)
    return s


def _prepare_objective(c, g, normal):
    nodes, edges, rows, first, coef = _tables(c)
    E, R, D = len(edges), len(rows), c["D"]
    s = dict(case=c, z=normal(nodes, D), v=normal(R, D), edge_ids=_ints(edges), row_parent=_ints(rows), row_first=_ints(first),
             row_coef=torch.tensor(coef, dtype=torch.float64).to(DEV), clip=1e-4, J=torch.empty(1, device=DEV), logp=torch.empty(E, device=DEV),
             grad=torch.empty(R, D, device=DEV), work=torch.empty(8 * (E * (D // 1024 + 2) + 1024), dtype=torch.uint8, device=DEV))
    # children near their step's mean, as a rollout leaves them: |z_child - mean|^2 h = about 1/2
    for r in range(R):
        a_z, a_v, h, _ = coef[r]
        m = a_z * s["z"][rows[r]] + a_v * s["v"][r]
        for e in range(first[r], first[r + 1]):
            s["z"][edges[e]] = m + math.sqrt(1.0 / (2.0 * h * D)) * normal(D)
    # what the rollout recorded: a policy that has moved by some clip ranges since, no edge on the border of the clip itself, where both sides are right
    move = normal(E) * 3e-4
    move = torch.where((move.abs() - 1e-4).abs() < 4e-6, move * 1.2, move).double()
    s["logp_old"] = torch.zeros(nodes, device=DEV)
    s["logp_old"][s["edge_ids"].long()] = (_exact_logp(s) - move).float()
    # advantages of kept edges: pruning keeps the ends of the rewards' order, more of the better one
    s["adv"] = (normal(nodes) * 1.0 + 0.4).clamp(-5, 5)
    return s


def _prepare_adamw(c, g, normal):
    sizes, (at, n) = _parameters(c), _places(c)
    s = dict(case=c, step=40, sizes=sizes, at=at, lr=1e-4, beta1=0.9, beta2=0.999, eps=1e-8, seed=1223627)
    live = torch.zeros(n, dtype=torch.bool, device=DEV)
    for a, (size, _) in zip(at, sizes):
        live[a:a + size] = True
    put = lambda x: torch.where(live, x, 0)  # noqa: E731  (between the tensors the buffers hold zeros)
    s["p"], s["g"] = put(normal(n) * 0.02), put(normal(n) * 1e-3 * (1 + 9 * torch.rand(n, generator=g, device=DEV) ** 8)).to(DTYPES[c["grads"]])
    s["copy"] = s["p"].to(torch.bfloat16) if c["copies"] else None
    # states after some steps: a mean of gradients below their scale, a second moment around its square
    m, v = put(normal(n) * 3e-4), put((normal(n) * 0.3 + 1).abs() * 1e-6)
    if c["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        s["m"], s["m_scale"] = _encode(m, 3, None)
        s["v"], s["v_scale"] = _encode(v.sqrt(), 4, None)
        s["m_value"], s["v_value"] = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    s["decay"] = [0.01 if is_matrix else 0.0 for _, is_matrix in sizes]
    if own:  # the optimizer's handle
        from paper_2509_06040_amd import binding as br
        part = lambda name: [s[name][a:a + k] for a, (k, _) in zip(at, sizes)]  # noqa: E731
        scales = lambda name: [s[name][a // 256:a // 256 + -(-k // 256)] for a, (k, _) in zip(at, sizes)]  # noqa: E731
        copies = [s["copy"][a:a + k] if is_matrix and c["copies"] else None for a, (k, is_matrix) in zip(at, sizes)]
        more = dict(m_scales=scales("m_scale"), v_scales=scales("v_scale")) if c["bits"] == 8 else {}
        s["optimizer"] = br.AdamW(part("p"), part("g"), part("m"), part("v"), copies=copies, weight_decay=s["decay"], lr=s["lr"], betas=(s["beta1"], s["beta2"]),
                                  eps=s["eps"], seed=s["seed"], step=s["step"], **more)
        if c["bits"] == 8:
            s["values"] = (part("m_value"), part("v_value"))
    return s


# ----------------------------------------------------------------------------------------------------------- the passes
def run(s):
    c = s["case"]
    return globals()["_%s_%s" % ("own" if own else "plain", c["kind"] + ("_" + {"fwd": "forward", "bwd": "backward"}[c["way"]] if "way" in c else ""))](s)


def _own_attention_forward(s):
    from paper_2509_06040_amd import binding as br
    br.attention_forward(s["q"], s["k"], s["v"], s["q_off"], s["k_off"], s["out"], s["lse"], s["work"])
    return s["out"], s["lse"]


def _own_attention_backward(s):
    from paper_2509_06040_amd import binding as br
    br.attention_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["q_off"], s["k_off"], s["dq"], s["dk"], s["dv"], s["work"])
    return s["dq"], s["dk"], s["dv"]


def _own_norm_forward(s):
    from paper_2509_06040_amd import binding as br
    br.layer_norm_forward(s["x"], s["mods"], s["shift_off"], s["scale_off"], s["row_off"], s["group"], s["out"], s["mean"], s["rstd"])
    return s["out"], s["mean"], s["rstd"]


def _own_norm_backward(s):
    from paper_2509_06040_amd import binding as br
    br.layer_norm_backward(s["dout"], s["x"], s["mean"], s["rstd"], s["mods"], s["shift_off"], s["scale_off"], s["row_off"], s["group"], s["residual"],
                           s["dx"], s["dmods"], s["work"])
    return s["dx"], s["dmods"]


def _own_objective(s):
    from paper_2509_06040_amd import binding as br
    br.grpo_backward(s["z"], s["v"], s["edge_ids"], s["row_parent"], s["row_first"], s["row_coef"], s["logp_old"], s["adv"], s["clip"], s["J"],
                     s["logp"], s["grad"], s["work"])
    return s["J"], s["logp"], s["grad"]


def _own_adamw(s):
    opt = s["optimizer"]
    opt.step()
    out = [s["p"]] + ([s["copy"]] if s["copy"] is not None else [])
    if s["case"]["bits"] == 32:
        return out + [s["m"], s["v"]]
    opt.state_values(*s["values"])
    return out + [s["m_value"], s["v_value"]]


def _padded(s):
    """Rows of the packed tokens by (document, place), what of it exists, and the document and place of each row."""
    at, there, docs, place = {}, {}, {}, {}
    for w, x in (("q", s["q"]), ("k", s["k"])):
        off = s[w + "_off"].long()
        n, most = off[1:] - off[:-1], s["most_" + w]
        i = torch.arange(most, device=DEV)
        there[w] = i < n[:, None]
        at[w] = torch.where(there[w], off[:-1, None] + i, 0)
        docs[w] = torch.repeat_interleave(torch.arange(len(n), device=DEV), n, output_size=x.shape[0])
        place[w] = torch.arange(x.shape[0], device=DEV) - off[:-1][docs[w]]
    return at, there, docs, place


def _spread(x, at, there, share=1):
    """[tokens, heads, d] -> [documents, heads * share, places, d] in 32 bits, zeros where nothing is."""
    if not x.shape[0]:
        x = x.new_zeros(1, *x.shape[1:])
    return torch.where(there[:, :, None, None], x[at].float(), 0).permute(0, 2, 1, 3).repeat_interleave(share, 1)


def _plain_scores(s, at, there):
    share = s["q"].shape[1] // s["k"].shape[1]
    q, k, v = _spread(s["q"], at["q"], there["q"]), _spread(s["k"], at["k"], there["k"], share), _spread(s["v"], at["k"], there["k"], share)
    scale = 1.0 / math.sqrt(q.shape[-1])
    x = torch.matmul(q, k.transpose(2, 3).contiguous()) * scale
    x = torch.where(there["k"][:, None, None, :], x, -math.inf)
    top = x.amax(3, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0, top))
    total = p.sum(3, keepdim=True)
    return q, k, v, p / torch.where(total == 0, 1, total), (top + torch.log(total)).squeeze(3), scale


def _plain_attention_forward(s):
    at, there, docs, place = _padded(s)
    q, k, v, p, lse, _ = _plain_scores(s, at, there)
    o = torch.matmul(p, v)
    return o[docs["q"], :, place["q"]].to(s["q"].dtype), lse[docs["q"], :, place["q"]].t().contiguous()


def _plain_attention_backward(s):
    at, there, docs, place = _padded(s)
    q, k, v, p, _, scale = _plain_scores(s, at, there)
    do = _spread(s["dout"], at["q"], there["q"])
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = p * (dp - (p * dp).sum(3, keepdim=True)) * scale
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3).contiguous(), q)
    kv = s["k"].shape[1]
    dk, dv = (x.view(x.shape[0], kv, -1, *x.shape[2:]).sum(2)[docs["k"], :, place["k"]] for x in (dk, dv))
    return tuple(x.to(s["q"].dtype) for x in (dq[docs["q"], :, place["q"]], dk, dv))


def _row_groups(s):
    off = s["row_off"].long()
    return torch.repeat_interleave(s["group"].long(), off[1:] - off[:-1], output_size=s["x"].shape[0])


def _plain_norm_forward(s):
    H, x = s["x"].shape[1], s["x"]
    rows = s["mods"][_row_groups(s)]
    mean = x.mean(1)
    rstd = 1 / torch.sqrt(((x - mean[:, None]) ** 2).mean(1) + 1e-6)
    y = (x - mean[:, None]) * rstd[:, None]
    y = y * (1 + rows[:, s["scale_off"]:s["scale_off"] + H]) + rows[:, s["shift_off"]:s["shift_off"] + H]
    return y.to(s["out"].dtype), mean, rstd


def _plain_norm_backward(s):
    H, x, dy = s["x"].shape[1], s["x"], s["dout"].float()
    groups = _row_groups(s)
    y = (x - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * (1 + s["mods"][:, s["scale_off"]:s["scale_off"] + H][groups])
    dx = s["residual"] + s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - y * (g * y).mean(1, keepdim=True))
    of = (groups == torch.arange(s["mods"].shape[0], device=DEV)[:, None]).float()
    s["dmods"][:, s["shift_off"]:s["shift_off"] + H] = torch.matmul(of, dy)
    s["dmods"][:, s["scale_off"]:s["scale_off"] + H] = torch.matmul(of, dy * y)
    return dx, s["dmods"]


def _plain_objective(s):
    E, R = s["edge_ids"].shape[0], s["row_parent"].shape[0]
    first, ids, coef = s["row_first"].long(), s["edge_ids"].long(), s["row_coef"].float()
    row = torch.repeat_interleave(torch.arange(R, device=DEV), first[1:] - first[:-1], output_size=E)
    mean = coef[:, 0:1] * s["z"][s["row_parent"].long()] + coef[:, 1:2] * s["v"]
    d = s["z"][ids] - mean[row]
    logp = coef[row, 3] - coef[row, 2] * (d * d).sum(1)
    ratio, a = torch.exp(logp - s["logp_old"][ids]), s["adv"][ids]
    free, held = ratio * a, torch.clamp(ratio, 1 - s["clip"], 1 + s["clip"]) * a
    w = torch.where(held < free, 0, free) * (-2 / E) * (coef[row, 2] * coef[row, 1])
    grad = torch.zeros_like(s["v"]).index_add_(0, row, d * w[:, None])
    return torch.minimum(free, held).mean().reshape(1), logp, grad


def _decode(code, scale, bits, sign):
    """Values of 8-bit codes: a sign where there is one, 4 bits of exponent, `bits` of mantissa; a code's number, without a leading one in the
    lowest exponent, times the scale of its block of 256."""
    c = code.int()
    low = c & 127 if sign else c
    e, f = low >> bits, low & ((1 << bits) - 1)
    x = torch.where(e > 0, (f + (1 << bits)) << (e - 1).clamp(min=0), f).float()
    x = torch.where((c & 128) > 0, -x, x) if sign else x
    return (x.view(-1, 256) * scale[:, None]).view(-1)


def _encode(x, bits, random16):
    """Codes and scales of blocks of 256 values.  The largest of a block takes the largest code; a value goes to one of its two neighbouring codes, up if
    the 16 random bits (0 .. 65535, as a fraction) reach over (None: to the nearest)."""
    most = float(((2 << bits) - 1) << 14)
    a = x.abs().view(-1, 256)
    top = a.amax(1)
    scale = top / torch.full_like(top, most)
    y = torch.clamp(a * torch.where(top > 0, torch.full_like(top, most) / torch.where(top > 0, top, 1), 0)[:, None], max=most).view(-1)
    e = (torch.frexp(y)[1] - 1 - bits).clamp(min=0)
    y = torch.ldexp(y, -e)
    y = torch.round(y) if random16 is None else torch.floor(y + random16.float() * (1 / 65536))
    code = (e << bits) + y.int()
    if bits == 3:
        code = code + torch.where(x < 0, 128, 0)
    return code.to(torch.uint8), scale


def _of_tensors(s, values, dtype, each=1):
    """A value of each tensor at every `each`-th of its elements."""
    ends = s["at"][1:] + [s["p"].shape[0]]
    return torch.cat([torch.full(((b - a) // each,), v, dtype=dtype, device=DEV) for a, b, v in zip(s["at"], ends, values)])


def _random_words(s):
    """The 32 random bits of every element: word i % 4 of Philox4x32-10 at (i / 4, tensor, step, 4), i an element's place in its tensor."""
    tensor, begin = _of_tensors(s, range(len(s["at"])), torch.int64, 4), _of_tensors(s, [a // 4 for a in s["at"]], torch.int64, 4)
    quad = torch.arange(len(begin), device=DEV) - begin
    x = [quad, tensor, torch.full_like(quad, s["step"]), torch.full_like(quad, 4)]
    k0, k1, low = s["seed"] & 0xFFFFFFFF, s["seed"] >> 32, 0xFFFFFFFF
    for _ in range(10):
        a, b = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [((b >> 32) & low) ^ x[1] ^ k0, b & low, ((a >> 32) & low) ^ x[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack(x, 1).view(-1)


def _plain_adamw(s):
    c = s["case"]
    s["step"] += 1
    decay = _of_tensors(s, [1.0 - s["lr"] * w for w in s["decay"]], torch.float32)
    g = s["g"].float()
    if c["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m = _decode(s["m"], s["m_scale"], 3, True)
        root = _decode(s["v"], s["v_scale"], 4, False)
        v = root * root
    m = m * s["beta1"] + g * (1.0 - s["beta1"])
    v = v * s["beta2"] + (g * (1.0 - s["beta2"])) * g
    root = torch.sqrt(v)
    change = m / (root * (1.0 / math.sqrt(1.0 - s["beta2"] ** s["step"])) + s["eps"])
    s["p"].copy_(s["p"] * decay - change * (s["lr"] / (1.0 - s["beta1"] ** s["step"])))
    out = [s["p"]]
    if s["copy"] is not None:
        of = _of_tensors(s, [is_matrix for _, is_matrix in s["sizes"]], torch.bool)
        s["copy"].copy_(torch.where(of, s["p"].to(torch.bfloat16), s["copy"]))
        out.append(s["copy"])
    if c["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return out + [s["m"], s["v"]]
    words = _random_words(s)
    for name, x, bits, r in (("m", m, 3, words & 0xFFFF), ("v", root, 4, words >> 16)):
        code, scale = _encode(x, bits, r)
        s[name].copy_(code)
        s[name + "_scale"].copy_(scale)
    root = _decode(s["v"], s["v_scale"], 4, False)
    return out + [_decode(s["m"], s["m_scale"], 3, True), root * root]


# ---------------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "norm": _exact_norm, "objective": _exact_objective, "adamw": _exact_adamw}[case["kind"]](s)


def _exact_attention(s):
    c, f = s["case"], torch.float64
    NH, NKV, d = c["heads"], c["kv_heads"], c["head_dim"]
    share, Tq, Tk = NH // NKV, s["q"].shape[0], s["k"].shape[0]
    o, lse = torch.zeros(Tq, NH, d, dtype=f, device=DEV), torch.full((NH, Tq), -math.inf, dtype=f, device=DEV)
    dq, dk, dv = torch.zeros_like(o), torch.zeros(Tk, NKV, d, dtype=f, device=DEV), torch.zeros(Tk, NKV, d, dtype=f, device=DEV)
    qo, ko = s["q_off"].tolist(), s["k_off"].tolist()
    for a, b, x, y in zip(qo, qo[1:], ko, ko[1:]):
        if a == b or x == y:
            continue
        for h in range(NH):
            q, k, v = s["q"][a:b, h].to(f), s["k"][x:y, h // share].to(f), s["v"][x:y, h // share].to(f)
            z = torch.mm(q, k.t().contiguous()) / math.sqrt(d)
            lse[h, a:b] = torch.logsumexp(z, 1)
            p = torch.exp(z - lse[h, a:b, None])
            o[a:b, h] = torch.mm(p, v)
            if c["way"] == "bwd":
                do = s["dout"][a:b, h].to(f)
                dv[x:y, h // share] += torch.mm(p.t().contiguous(), do)
                g = p * (torch.mm(do, v.t().contiguous()) - (do * o[a:b, h]).sum(1, keepdim=True)) / math.sqrt(d)
                dq[a:b, h] = torch.mm(g, k)
                dk[x:y, h // share] += torch.mm(g.t().contiguous(), q)
    return (o, lse) if c["way"] == "fwd" else (dq, dk, dv)


def _exact_norm(s):
    H, R, G = s["x"].shape[1], s["x"].shape[0], s["mods"].shape[0]
    off, group = s["row_off"].tolist(), s["group"].tolist()
    x, mods = s["x"].double(), s["mods"].double()
    if s["case"]["way"] == "fwd":
        out = torch.empty(R, H, dtype=torch.float64, device=DEV)
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = (var + 1e-6) ** -0.5
        for a, b, k in zip(off, off[1:], group):
            out[a:b] = torch.addcmul(mods[k, s["shift_off"]:][:H], (x[a:b] - mean[a:b, None]) * rstd[a:b, None], 1 + mods[k, s["scale_off"]:][:H])
        return out, mean, rstd
    # the rows' own statistics, as the forward pass gave them, are inputs
    n = (x - s["mean"].double()[:, None]) * s["rstd"].double()[:, None]
    dy, dx, dmods = s["dout"].double(), s["residual"].double(), torch.zeros(mods.shape, dtype=torch.float64, device=DEV)
    for a, b, k in zip(off, off[1:], group):
        y = dy[a:b] * (1 + mods[k, s["scale_off"]:][:H])
        dx[a:b] += s["rstd"][a:b, None].double() * (y - y.sum(1, keepdim=True) / H - n[a:b] * ((y * n[a:b]).sum(1, keepdim=True) / H))
        dmods[k, s["shift_off"]:s["shift_off"] + H] += dy[a:b].sum(0)
        dmods[k, s["scale_off"]:s["scale_off"] + H] += (dy[a:b] * n[a:b]).sum(0)
    return dx, dmods


def _exact_logp(s):
    first, ids, rows = s["row_first"].tolist(), s["edge_ids"].tolist(), s["row_parent"].tolist()
    coef, out = s["row_coef"].tolist(), torch.empty(len(ids), dtype=torch.float64, device=DEV)
    for r, (a_z, a_v, h, c0) in enumerate(coef):
        m = a_z * s["z"][rows[r]].double() + a_v * s["v"][r].double()
        for e in range(first[r], first[r + 1]):
            out[e] = c0 - h * torch.sum((s["z"][ids[e]].double() - m) ** 2)
    return out


def _exact_objective(s):
    first, ids, rows, coef = s["row_first"].tolist(), s["edge_ids"].tolist(), s["row_parent"].tolist(), s["row_coef"].tolist()
    logp = _exact_logp(s)
    new, old, adv = logp.tolist(), s["logp_old"].tolist(), s["adv"].tolist()
    J, grad = 0.0, torch.zeros(s["v"].shape, dtype=torch.float64, device=DEV)
    for r, (a_z, a_v, h, _) in enumerate(coef):
        m = a_z * s["z"][rows[r]].double() + a_v * s["v"][r].double()
        for e in range(first[r], first[r + 1]):
            ratio, a = math.exp(new[e] - old[ids[e]]), adv[ids[e]]
            inside = min(max(ratio, 1 - s["clip"]), 1 + s["clip"]) * a
            J += min(ratio * a, inside) / len(ids)
            if inside >= ratio * a:  # d(-J)/dv = -ratio A / n * dlogp/dv
                grad[r] -= ratio * a / len(ids) * 2 * h * a_v * (s["z"][ids[e]].double() - m)
    return torch.tensor([J], dtype=torch.float64), logp, grad


def _exact_adamw(s):
    c = s["case"]
    s["step"] += 1
    t, b1, b2 = s["step"], s["beta1"], s["beta2"]
    if c["bits"] == 8:
        table = [torch.tensor([(-1 if sign and code > 127 else 1) * ((code & 127 if sign else code) if (code & 127 if sign else code) < (2 << bits) else
                               ((1 << bits) + (code & ((1 << bits) - 1))) * 2.0 ** (((code & 127 if sign else code) >> bits) - 1)) for code in range(256)],
                              dtype=torch.float64, device=DEV) for bits, sign in ((3, True), (4, False))]
        m = (table[0][s["m"].int()].view(-1, 256) * s["m_scale"].double()[:, None]).view(-1)
        v = (table[1][s["v"].int()].view(-1, 256) * s["v_scale"].double()[:, None]).view(-1) ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    p, g = s["p"].double(), s["g"].double()
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    copy = None if s["copy"] is None else s["copy"].double()
    for i, (a, (n, is_matrix)) in enumerate(zip(s["at"], s["sizes"])):
        x = slice(a, a + n)
        p[x] -= s["lr"] * (s["decay"][i] * p[x] + m[x] / (1 - b1 ** t) / ((v[x] / (1 - b2 ** t)) ** 0.5 + s["eps"]))
        if copy is not None and is_matrix:
            copy[x] = p[x]
    out = [p] + ([copy] if copy is not None else [])
    if c["bits"] == 32:
        return out + [m, v]
    words = _random_words(s)
    for x, bits, r, square in ((m, 3, words & 0xFFFF, False), (v ** 0.5, 4, words >> 16, True)):
        most = ((2 << bits) - 1) * 2.0 ** 14
        top = x.abs().view(-1, 256).amax(1).repeat_interleave(256)
        y = torch.where(top > 0, x.abs() / torch.where(top > 0, top, 1) * most, 0)
        gap = torch.exp2(torch.floor(torch.log2(y.clamp(min=1.0))) - bits).clamp(min=1.0)
        y = (torch.floor(y / gap + r / 65536.0) * gap).clamp(max=most) * top / most * torch.sign(x)
        out.append(y ** 2 if square else y)
    return out
