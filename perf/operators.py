"""Operators around the sparse layer in a training step, as cases that can be timed and compared.

Three operators: the block norm (norm of a block's output, gate, residual add and
the next norm in one pass, forward and backward), the load-balance loss with the
experts' demand, and AdamW over many tensors with states in 32 or 8 bits. `run`
computes them through the library where `own` is true and in elementary torch
operations where it is not; `exact` is the definition in 64 bits. Shapes are
those of the benchmark's workloads and of neighbouring widths and batches.
"""
from __future__ import annotations

import math

import torch

own = False  # True: through the library's entry points

DEV = "cuda"
BLOCK = 128  # elements that share one scale of an 8-bit state


# ------------------------------------------------------------------ cases

def _norm(name, kind, tokens, d, **more):
    """kind: norm_fwd | norm_bwd; pre, post: none | rms | layer."""
    c = dict(name=name, kind=kind, tokens=tokens, groups=1, d=d, dtype="bf16", stream="bf16",
             dh="f32", pre="layer", post="none", bias=True, gate=True, drop=0.0)
    c.update(more)
    return c


def _balance(name, groups, group_tokens, experts, k, **more):
    c = dict(name=name, kind="balance", groups=groups, group_tokens=group_tokens, experts=experts,
             k=k, noise=True, padding=0.0, hot=0)
    c.update(more)
    return c


def _adamw(name, tensors, d, f, experts, blocks, **more):
    """tensors: vectors (norm weights and biases) | blocks (those, attention-free
    sparse blocks: router and experts too). state: f32 | 8bit | mixed (8 bits
    for tensors of 16384 elements or more)."""
    c = dict(name=name, kind="adamw", tensors=tensors, d=d, f=f, experts=experts, blocks=blocks,
             dtype="bf16", grad="f32", state="f32", clip="none")
    c.update(more)
    return c


def listed():
    return [
        # One 224-px image through a ViT-B/16 block, forward: launch latency.
        _norm("norm_fwd_one_image", "norm_fwd", 197, 768),
        # The headline batch (ViT-L/16 at 384 px) with drop-path, forward.
        _norm("norm_fwd_vitl16", "norm_fwd", 36928, 1024, drop=0.1),
        # The same, backward: the layer hands its input gradient over in f32.
        _norm("norm_bwd_vitl16", "norm_bwd", 36928, 1024, drop=0.1),
        # The small f32 layer, backward, norms on both sides of the block.
        _norm("norm_bwd_tiny_f32", "norm_bwd", 788, 192, dtype="f32", stream="f32", post="layer"),
        # A wide model with RMS norms on both sides, an f32 residual stream and a
        # gate for each sequence; an odd number of tokens.
        _norm("norm_bwd_wide_rms", "norm_bwd", 7 * 1171, 4096, groups=7, stream="f32", dh="bf16",
              pre="rms", post="rms", bias=False),
        # One image's gate (8 experts).
        _balance("balance_one_image", 1, 197, 8, 2),
        # The headline's gate: 32 experts, four of them hot.
        _balance("balance_vitl16", 1, 36928, 32, 2, hot=4),
        # A long batch of ragged sequences with padding and many experts.
        _balance("balance_ragged_e64", 61, 4093, 64, 6, noise=False, padding=0.2, hot=3),
        # Norm weights and biases of a small f32 model: many tiny tensors.
        _adamw("adamw_vectors_f32", "vectors", 192, 768, 8, 12, dtype="f32"),
        # One ViT-B/16 layer of eight experts with f32 states and an active
        # gradient-norm clip.
        _adamw("adamw_vitb16_clip", "blocks", 768, 3072, 8, 1, clip="active"),
        # Every tensor of twelve narrow blocks with odd widths, bf16 gradients,
        # large tensors in 8 bits and small ones in 32, a clip that is not reached.
        _adamw("adamw_blocks_mixed", "blocks", 328, 1304, 6, 12, grad="bf16", state="mixed",
               clip="idle"),
        # The headline layer's 268 million expert weights with 8-bit states.
        _adamw("adamw_vitl16_8bit", "blocks", 1024, 4096, 32, 1, state="8bit"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case of the listed ranges: 1 to 40 000 tokens and widths 64 to
    8192 for the norms, 16 to 260 000 tokens and 2 to 64 experts for the loss,
    hundreds to 270 million parameters for AdamW."""
    kind = rng.choice(["norm_fwd", "norm_fwd", "norm_bwd", "norm_bwd", "norm_bwd", "balance",
                       "balance", "adamw", "adamw", "adamw"])
    while True:
        if kind == "balance":
            groups = rng.choice([1, 1, 1, 2, 5, 17, 64])
            tokens = max(1, _log(rng, 16, 260000) // groups)
            experts = rng.choice([2, 4, 6, 8, 12, 16, 24, 32, 48, 64])
            k = min(experts, rng.choice([1, 2, 2, 2, 3, 4, 6, 8]))
            if groups * tokens * experts > 61 * 4093 * 64:
                continue
            c = _balance("", groups, tokens, experts, k, noise=rng.random() < 0.5,
                         padding=rng.choice([0.0, 0.0, 0.1, 0.5]), hot=rng.choice([0, 1, 2]))
        elif kind == "adamw":
            d = 8 * _log(rng, 8, 128)
            f = 8 * round(d * rng.choice([2, 3, 4, 4]) / 8)
            experts, blocks = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([1, 1, 2, 3, 6, 12, 24])
            tensors = rng.choice(["vectors", "blocks", "blocks", "blocks"])
            size = blocks * experts * 2 * d * f
            dtype = rng.choice(["f32", "bf16", "bf16"])
            state = rng.choice(["f32", "8bit", "mixed"])
            c = _adamw("", tensors, d, f, experts, blocks, dtype=dtype, state=state,
                       grad="f32" if dtype == "f32" else rng.choice(["f32", "bf16"]),
                       # an active clip makes gradients differ in the last bit with the order of
                       # the norm's sum, and a rounding to 8 bits could fall to either side of it
                       clip=rng.choice(["none", "idle", "active"] if state == "f32"
                                       else ["none", "idle"]))
            if tensors == "blocks" and (size > 2 * 32 * 1024 * 4096 or work(c)["bytes"] > 6.4e9):
                continue
        else:
            d = 8 * _log(rng, 8, 1024)
            groups = rng.choice([1, 1, 1, 3, 16])
            tokens = groups * max(1, _log(rng, 1, 40000) // groups)
            if tokens * d > 36928 * 1024:
                continue
            dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
            c = _norm("", kind, tokens, d, groups=groups, dtype=dtype,
                      stream="f32" if dtype == "f32" else rng.choice(["bf16", "f32"]),
                      dh="f32" if dtype == "f32" else rng.choice(["f32", "bf16"]),
                      pre=rng.choice(["rms", "layer"]), post=rng.choice(["none", "rms", "layer"]),
                      bias=rng.random() < 0.5, gate=rng.random() < 0.7,
                      drop=rng.choice([0.0, 0.0, 0.2]))
        if 3072 in (c.get("d"), c.get("tokens"), c.get("group_tokens")):
            continue
        del c["name"]
        return c


def _t(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _bytes(name):
    return 2 if name == "bf16" else 4


def work(c):
    if c["kind"] == "adamw":
        sizes = _sizes(c)
        small = [n for n in sizes if not _is_8bit(c, n)]
        n, n32 = sum(sizes), sum(small)
        n8 = n - n32
        weight = 8 + (2 if c["dtype"] == "bf16" else 0)  # read, written, and the bf16 copy
        # 8-bit states: read, written, and their values handed out in bf16
        return dict(bytes=n * (weight + _bytes(c["grad"])) + 16 * n32 + 8 * n8 + 4 * n8 // BLOCK,
                    flops=14 * n)
    if c["kind"] == "balance":
        n = c["groups"] * c["group_tokens"]
        rows = n * c["experts"] * 4
        return dict(bytes=rows * (4 if c["noise"] else 3) + n * c["k"] * 4
                    + (n if c["padding"] else 0), flops=8 * n * c["experts"])
    n, s, a = c["tokens"] * c["d"], _bytes(c["stream"]), _bytes(c["dtype"])
    stats = 8 * c["tokens"] * (2 if c["post"] != "none" else 1)
    a *= 2 - c["drop"]  # a dropped token's block output is not read
    if c["kind"] == "norm_fwd":
        return dict(bytes=round(n * (2 * s + a)) + stats, flops=14 * n)
    return dict(bytes=round(n * (3 * s + a + _bytes(c["dh"]))) + stats, flops=30 * n)


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def _prepare_norm(c, seed):
    g, n, d, G = _gen(seed), c["tokens"], c["d"], c["groups"]
    act, res = _t(c["dtype"]), _t(c["stream"])
    s = dict(case=c)
    # the stream grows along the depth and has a few strong channels
    loud = 1 + 4 * (torch.rand(d, device=DEV, generator=g) < 0.01).float()
    s["x"] = (1.5 * _randn(g, n, d) * loud + 0.2).to(res)
    s["y"] = (0.7 * _randn(g, n, d)).to(act)
    vector = lambda mean: (mean + 0.1 * _randn(g, d)).to(act)  # noqa: E731
    s["pre_w"], s["pre_b"] = vector(1.0), vector(0.0) if c["bias"] and c["pre"] == "layer" else None
    s["post_w"] = vector(1.0) if c["post"] != "none" else None
    s["post_b"] = vector(0.0) if c["bias"] and c["post"] == "layer" else None
    s["gate"] = (0.5 + 0.2 * _randn(g, G, d)).to(act) if c["gate"] else None
    keep = 1 - c["drop"]  # drop-path: a dropped token's block is skipped, the others scaled up
    s["row_scale"] = (torch.rand(n, device=DEV, generator=g) < keep).float() / keep \
        if c["drop"] else None
    if c["kind"] == "norm_bwd":  # s["x"] stands for the forward's output here
        s["pre_stats"] = _stats(s["x"].float(), c["pre"])
        s["post_stats"] = _post_stats(s, s["y"].float()) if c["post"] != "none" else None
        s["dx_out"] = _randn(g, n, d).to(res)
        s["dh"] = (0.3 * _randn(g, n, d)).to(_t(c["dh"]))
    new = lambda dt, *shape: torch.empty(*shape, dtype=dt, device=DEV)  # noqa: E731
    like = lambda w, *shape: None if w is None else new(torch.float32, *shape)  # noqa: E731
    if c["kind"] == "norm_fwd":
        s["out"] = dict(x_out=new(res, n, d), h=new(act, n, d),
                        pre_stats=new(torch.float32, n, 2), post_stats=like(s["post_w"], n, 2))
    else:
        s["out"] = dict(dx=new(res, n, d), dy=new(act, n, d), dpre_w=like(s["pre_w"], d),
                        dpre_b=like(s["pre_b"], d), dpost_w=like(s["post_w"], d),
                        dpost_b=like(s["post_b"], d), dgate=like(s["gate"], G, d))
    return s


def _prepare_balance(c, seed):
    g = _gen(seed)
    G, E, k = c["groups"], c["experts"], c["k"]
    n = G * c["group_tokens"]
    s = dict(case=c)
    s["logits"] = _randn(g, n, E)
    s["bias"] = torch.where(torch.arange(E, device=DEV) < c["hot"], 2.0, 0.0) if c["hot"] else None
    s["noise"] = _randn(g, n, E) / math.sqrt(E) if c["noise"] else None
    z = _gate_logits(s)
    s["probs"] = torch.softmax(z, 1)
    s["expert_idx"] = torch.topk(z, k, 1).indices.to(torch.int32)
    s["mask"] = (torch.rand(n, device=DEV, generator=g) >= c["padding"]).to(torch.uint8) \
        if c["padding"] else None
    s["w_balance"], s["w_z"] = 0.01, 0.001
    s["out"] = dict(losses=torch.empty(G, 2, device=DEV),
                    demand=torch.empty(G, E, dtype=torch.int32, device=DEV),
                    mean_probs=torch.empty(G, E, device=DEV), dlogits=torch.empty(n, E, device=DEV))
    return s


def _sizes(c):
    d, f, E = c["d"], c["f"], c["experts"]
    vectors = [d, d, d, E * f, E * d]
    if c["tensors"] == "vectors":
        return c["blocks"] * [d, d, d, f, d]
    return c["blocks"] * (vectors + [E * d, E * d * f, E * d * f])


def _is_8bit(c, n):
    return c["state"] == "8bit" or (c["state"] == "mixed" and n >= 16384)


def _decayed(n):
    return n >= 16384


def _prepare_adamw(c, seed):
    """Tensors are parts of flat buffers, each part a whole number of state
    blocks long, as a program with flat optimizer buffers has them: one flat
    set for tensors with 32-bit states and one for those with 8-bit ones."""
    g = _gen(seed)
    s = dict(case=c, step=100, seed=seed & 0xFFFFFFFF,
             hyper=dict(lr=1e-4, beta1=0.9, beta2=0.999, eps=1e-8))
    s["sets"] = {}
    for kind in ("f32", "8bit"):
        sizes = [n for n in _sizes(c) if _is_8bit(c, n) == (kind == "8bit")]
        if sizes:
            s["sets"][kind] = _flat_set(c, g, sizes, kind)
    s["norm_out"] = torch.empty(2, device=DEV)
    # the norm is about 1e-3 sqrt(n): far below or far above what is allowed
    s["max_norm"] = dict(none=math.inf, idle=1e6, active=1e-2)[c["clip"]]
    return s


def _flat_set(c, g, sizes, kind):
    slots = torch.tensor([-(-n // BLOCK) * BLOCK for n in sizes])
    ends = slots.cumsum(0)
    total = int(ends[-1])
    starts = (ends - slots).tolist()
    tensor = torch.repeat_interleave(torch.arange(len(sizes), device=DEV), slots.to(DEV),
                                     output_size=total)
    place = torch.arange(total, device=DEV) - (ends - slots).to(DEV)[tensor]
    live = place < torch.tensor(sizes, device=DEV)[tensor]
    rate = [0.05 if _decayed(n) else 0.0 for n in sizes]
    decay = torch.tensor(rate, device=DEV)[tensor] * live
    del tensor, place
    # parameters as they are drawn at the start; gradients whose size varies over
    # blocks of channels, with a few outliers; moments of earlier gradients
    size = 1e-3 * torch.exp(0.7 * _randn(g, total // BLOCK, 1)).expand(-1, BLOCK).reshape(-1)
    grad = _randn(g, total) * size * live
    master = 0.02 * _randn(g, total) * live
    m = 0.3 * size * _randn(g, total) * live
    v = size.square() * torch.exp(0.5 * _randn(g, total)) * live
    q = dict(sizes=sizes, starts=starts, kind=kind, decay=decay, grad=grad.to(_t(c["grad"])),
             master=master, param=master.to(torch.bfloat16) if c["dtype"] == "bf16" else None)
    if kind == "f32":
        q["m"], q["v"] = m, v
    else:  # states that 8 bits hold: any code, below a scale for each block
        q["m"] = _random_codes(g, total, 0x30, 0x78, True) * live
        q["v"] = _random_codes(g, total, 0xC0, 0xF8, False) * live
        high = torch.floor(torch.log2(size[::BLOCK])).to(torch.int32) + 127
        q["m_scale"] = high.to(torch.uint8)
        q["v_scale"] = (2 * (high - 127) + 128).to(torch.uint8)
        q["m_value"] = torch.empty(total, dtype=torch.bfloat16, device=DEV)
        q["v_value"] = torch.empty(total, dtype=torch.bfloat16, device=DEV)
    return q


def _random_codes(g, n, lo, hi, signed):
    code = torch.randint(lo, hi, (n,), device=DEV, generator=g, dtype=torch.int32)
    if signed:
        code += 128 * torch.randint(0, 2, (n,), device=DEV, generator=g, dtype=torch.int32)
    return code.to(torch.uint8)


def prepare(case, seed):
    if case["kind"] == "adamw":
        s = _prepare_adamw(case, seed)
    else:
        s = _prepare_balance(case, seed) if case["kind"] == "balance" else _prepare_norm(case, seed)
    if own:
        _handles(s)
    return s


# ------------------------------------------------------------------ through the library

def _handles(s):
    """The shape, workspace and plan that a program makes once."""
    from paper_2608_16188_amd import vmoe as V
    from paper_2608_16188_amd import vmoe_train as T
    c = s["case"]
    if c["kind"] == "adamw":
        tensors = []
        for q in s["sets"].values():
            for n, at in zip(q["sizes"], q["starts"]):
                part = slice(at, at + n)
                scales = slice(at // BLOCK, -(-(at + n) // BLOCK))
                bits8 = q["kind"] == "8bit"
                tensors.append(T.AdamWTensor(
                    param=q["master"][part] if q["param"] is None else q["param"][part],
                    master=None if q["param"] is None else q["master"][part],
                    grad=q["grad"][part], m=q["m"][part], v=q["v"][part],
                    m_scale=q["m_scale"][scales] if bits8 else None,
                    v_scale=q["v_scale"][scales] if bits8 else None,
                    weight_decay=0.05 if _decayed(n) else 0.0, index0=at))
        s["plan"] = T.AdamWPlan(tensors)
        s["ws"] = torch.empty(T.vmoe_grad_norm_workspace_bytes(s["plan"]), dtype=torch.uint8,
                              device=DEV)
        return
    if c["kind"] == "balance":
        s["shape"] = V.make_shape(c["groups"] * c["group_tokens"], c["groups"], 64, 64,
                                  c["experts"], c["k"], 1.0, V.VMOE_F32)
        ws = T.vmoe_load_balance_loss_workspace_bytes(s["shape"])
    else:
        dt = dict(bf16=V.VMOE_BF16, f32=V.VMOE_F32)
        kind = dict(none=T.VMOE_NORM_NONE, rms=T.VMOE_NORM_RMS, layer=T.VMOE_NORM_LAYER)
        s["shape"] = T.make_norm_shape(c["tokens"], c["d"], dt[c["dtype"]], n_groups=c["groups"],
                                       stream_dtype=dt[c["stream"]], dh_dtype=dt[c["dh"]],
                                       pre_norm=kind[c["pre"]], post_norm=kind[c["post"]],
                                       eps=1e-6, residual_scale=1.0, branch_scale=1.0)
        ws = T.vmoe_block_norm_bwd_workspace_bytes(s["shape"]) if c["kind"] == "norm_bwd" else 0
    s["ws"] = torch.empty(ws, dtype=torch.uint8, device=DEV)


def _run_own(s):
    from paper_2608_16188_amd import vmoe_train as T
    c, o = s["case"], s["out"] if "out" in s else None
    if c["kind"] == "norm_fwd":
        T.vmoe_block_norm_fwd(s["shape"], s["x"], s["y"], s["post_w"], s["post_b"], s["gate"],
                              s["row_scale"], s["pre_w"], s["pre_b"], o["x_out"], o["h"],
                              o["post_stats"], o["pre_stats"])
        return _present(o)
    if c["kind"] == "norm_bwd":
        T.vmoe_block_norm_bwd(s["shape"], s["dx_out"], s["dh"], s["x"], s["y"], s["post_w"],
                              s["post_b"], s["gate"], s["row_scale"], s["pre_w"], s["post_stats"],
                              s["pre_stats"], o["dx"], o["dy"], o["dpost_w"], o["dpost_b"],
                              o["dgate"], o["dpre_w"], o["dpre_b"], s["ws"])
        return _present(o)
    if c["kind"] == "balance":
        T.vmoe_load_balance_loss(s["shape"], s["logits"], s["bias"], s["noise"], s["probs"],
                                 s["expert_idx"], s["mask"], s["w_balance"], s["w_z"], o["losses"],
                                 o["demand"], o["mean_probs"], o["dlogits"], s["ws"])
        return o
    s["step"] += 1
    clip = None
    if c["clip"] != "none":
        clip = s["norm_out"]
        T.vmoe_grad_norm(s["plan"], s["max_norm"], clip, s["ws"])
    T.vmoe_adamw(s["plan"], **s["hyper"], step=s["step"], seed=s["seed"], clip=clip)
    if "8bit" in s["sets"]:
        q = s["sets"]["8bit"]
        T.vmoe_adamw_state_values(q["m"], q["m_scale"], True, q["m_value"])
        T.vmoe_adamw_state_values(q["v"], q["v_scale"], False, q["v_value"])
    return _adamw_outputs(s, clip)


def _present(d):
    return {k: t for k, t in d.items() if t is not None}


def _adamw_outputs(s, clip):
    """The updated buffers; 8-bit states as the values they stand for."""
    out = {kind: _present(dict(param=q["param"], master=q["master"],
                               m=q["m"] if kind == "f32" else q["m_value"],
                               v=q["v"] if kind == "f32" else q["v_value"]))
           for kind, q in s["sets"].items()}
    if clip is not None:
        out["norm"] = clip[:1]
    return out


# ------------------------------------------------------------------ plain form

def _stats(x, kind):
    """[N, 2]: mean (0 for rms) and the reciprocal deviation."""
    mean = x.mean(1) if kind == "layer" else torch.zeros_like(x[:, 0])
    var = (x - mean[:, None]).square().mean(1)
    return torch.stack([mean, 1 / torch.sqrt(var + 1e-6)], 1)


def _post_stats(s, y):
    """Those of the block's output; 0 for a dropped token, whose output is not looked at."""
    r = _stats(y, s["case"]["post"])
    return r if s["row_scale"] is None else torch.where(s["row_scale"][:, None] != 0, r, 0.0)


def _unit(x, stats):
    return (x - stats[:, :1]) * stats[:, 1:]


def _affine(n, w, b):
    n = n * w if w is not None else n
    return n + b if b is not None else n


def _by_token(gate, n):
    """[G, d] -> [N, d]: each group's row for its tokens."""
    return gate.repeat_interleave(n // gate.shape[0], 0) if gate.shape[0] > 1 else gate


def _wide(s, to, *names):
    return [None if s[k] is None else s[k].to(to) for k in names]


def _norm_fwd(s, to):
    """The forward in the arithmetic of type `to`, unrounded."""
    c = s["case"]
    x, y, post_w, post_b, gate, row, pre_w, pre_b = _wide(
        s, to, "x", "y", "post_w", "post_b", "gate", "row_scale", "pre_w", "pre_b")
    out = {}
    if c["post"] != "none":
        out["post_stats"] = _post_stats(s, y)
        y = _affine(_unit(y, out["post_stats"]), post_w, post_b)
    if gate is not None:
        y = y * _by_token(gate, c["tokens"])
    if row is not None:
        y = y * row[:, None]
    out["x_out"] = x + y
    out["pre_stats"] = _stats(out["x_out"], c["pre"])
    out["h"] = _affine(_unit(out["x_out"], out["pre_stats"]), pre_w, pre_b)
    return out


def _norm_grad(dn, n, stats, kind):
    """Gradient at the input of a norm from dn, the gradient at its unit output n."""
    dot = (dn * n).mean(1, keepdim=True)
    if kind == "layer":
        dn = dn - dn.mean(1, keepdim=True)
    return (dn - n * dot) * stats[:, 1:]


def _norm_bwd(s, to):
    c = s["case"]
    x, y, post_w, post_b, gate, row, pre_w, pre_b, dx_out, dh, pre_stats, post_stats = _wide(
        s, to, "x", "y", "post_w", "post_b", "gate", "row_scale", "pre_w", "pre_b", "dx_out",
        "dh", "pre_stats", "post_stats")
    out = {}
    n = _unit(x, pre_stats)
    out["dpre_w"] = (dh * n).sum(0)
    if pre_b is not None:
        out["dpre_b"] = dh.sum(0)
    G = dx_out + _norm_grad(dh * pre_w, n, pre_stats, c["pre"])
    out["dx"] = G
    if row is not None:
        G = G * row[:, None]
    ny = _unit(y, post_stats) if c["post"] != "none" else y
    if gate is not None:
        out["dgate"] = (G * _affine(ny, post_w, post_b)).view(c["groups"], -1, c["d"]).sum(1)
        G = G * _by_token(gate, c["tokens"])
    if c["post"] != "none":
        out["dpost_w"] = (G * ny).sum(0)
        if post_b is not None:
            out["dpost_b"] = G.sum(0)
        G = _norm_grad(G * post_w, ny, post_stats, c["post"])
    out["dy"] = G
    return out


def _gate_logits(s):
    z = s["logits"]
    z = z + s["bias"] if s["bias"] is not None else z
    return z + s["noise"] if s["noise"] is not None else z


def _balance_loss(s, to):
    c = s["case"]
    G, E, k = c["groups"], c["experts"], c["k"]
    z, probs = _gate_logits(s).to(to), s["probs"].to(to)
    live = torch.ones_like(z[:, 0]) if s["mask"] is None else (s["mask"] != 0).to(to)
    top = z.max(1, keepdim=True).values
    lse = (top + torch.log(torch.exp(z - top).sum(1, keepdim=True)))[:, 0]
    chosen = s["expert_idx"][:, :, None] == torch.arange(E, device=z.device)
    demand = (chosen.sum(1) * live[:, None].to(torch.int64)).view(G, -1, E).sum(1)
    n = live.view(G, -1).sum(1)
    n1 = torch.clamp(n, min=1)[:, None]
    f = demand.to(to) / (k * n1)
    mean_probs = (probs * live[:, None]).view(G, -1, E).sum(1) / n1
    loss = E * (f * mean_probs).sum(1)
    z_loss = (lse.square() * live).view(G, -1).sum(1) / n1[:, 0]
    ft = _by_token(f, probs.shape[0])
    per_token = _by_token(live.new_ones(G, 1) / n1, probs.shape[0]) * live[:, None]
    dlogits = per_token * probs * (s["w_balance"] * E * (ft - (ft * probs).sum(1, keepdim=True))
                                   + 2 * s["w_z"] * lse[:, None])
    return dict(losses=torch.stack([loss, z_loss], 1), demand=demand.to(torch.int32),
                mean_probs=mean_probs, dlogits=dlogits)


# 8-bit states. A block of 128 values has one scale, a power of two 2^(e - 127)
# with e held in a byte. Codes count 3 mantissa bits and 4 (m, beside a sign) or 5
# (v) exponent bits below the scale; the lowest exponent is linear down to 0.

def _code_values(low):
    """The 2^(bits) values of the codes without sign; low: exponent of code 8."""
    code = torch.arange(256 if low == -30 else 128, device=DEV)
    exponent, mantissa = code >> 3, (code & 7).to(torch.float64)
    v = torch.where(exponent > 0, (8 + mantissa) * 2.0 ** (torch.clamp(exponent, min=1) - 1),
                    mantissa) * 2.0 ** (low - 3)
    return v if low == -30 else torch.cat([v, -v])


def _power(e):
    """2^e in f32 from its bits, -126 <= e <= 127."""
    return ((e + 127) << 23).view(torch.float32)


def _decode(code, scale, low):
    table = _code_values(low).to(torch.float32)
    return (table[code.to(torch.int32)].view(-1, BLOCK)
            * _power(scale.to(torch.int32) - 127)[:, None]).view(-1)


def _encode(x, r, low):
    """Codes, scales and values of x >= 0 or of |x|; r in (0, 1) rounds: up where
    it reaches over what is cut off."""
    blocks = x.view(-1, BLOCK)
    top = blocks.amax(1).view(torch.int32)
    e = (top + 0xFFFFF) >> 23
    unit = _power(127 - e)[:, None] * blocks  # in [0, 2)
    exponent = torch.clamp((unit.view(torch.int32) >> 23) - 127, min=low)
    count = torch.floor(unit * _power(3 - exponent) + r.view(-1, BLOCK))
    if low == -30:  # what is above 0 stays above 0
        count = torch.where((unit > 0) & (count == 0), 1.0, count)
    value = count * _power(exponent - 3)
    # a count of 16 is the next exponent's 8
    code = (exponent - low) * 8 + count.to(torch.int32)
    return code.view(-1), e.to(torch.uint8), (value * _power(e - 127)[:, None]).view(-1)


def _mix(x):
    """32 bits of x, mixed (whole numbers in 64 bits, masked to 32)."""
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random(n, step, seed):
    """Two numbers in (0, 1) for each element from the step, the seed and its index."""
    key = _mix(seed ^ _mix((step * 0x9E3779B1) & 0xFFFFFFFF))
    index = torch.arange(n, device=DEV, dtype=torch.int64)
    bits = _mix(((index * 0x9E3779B1) & 0xFFFFFFFF) ^ key)
    half = 0.5 / 65536
    return (bits & 0xFFFF).to(torch.float32) / 65536 + half, \
        (bits >> 16).to(torch.float32) / 65536 + half


def _adamw_step(q, hyper, step, scale, to):
    """New m, v and master weights of one flat set in the arithmetic of type `to`."""
    b1, b2 = hyper["beta1"], hyper["beta2"]
    m, v = q["m"], q["v"]
    if q["kind"] == "8bit":
        m, v = _decode(m, q["m_scale"], -14), _decode(v, q["v_scale"], -30)
    g = q["grad"].to(to)
    g = g * scale if scale is not None else g
    m = m.to(to) * b1 + g * (1 - b1)
    v = v.to(to) * b2 + g * g * (1 - b2)
    c1, c2 = 1 / (1 - b1 ** step), 1 / math.sqrt(1 - b2 ** step)
    p = q["master"].to(to)
    p = p - hyper["lr"] * (m * c1 / (torch.sqrt(v) * c2 + hyper["eps"]) + q["decay"].to(to) * p)
    return m, v, p


def _adamw_set(q, s, scale):
    m, v, p = _adamw_step(q, s["hyper"], s["step"], scale, torch.float32)
    q["master"].copy_(p)
    if q["param"] is not None:
        q["param"].copy_(p)
    if q["kind"] == "f32":
        q["m"].copy_(m)
        q["v"].copy_(v)
        return
    rm, rv = _random(m.numel(), s["step"], s["seed"])
    code, scale8, value = _encode(m.abs(), rm, -14)
    q["m"].copy_(torch.where(m < 0, code + 128, code))
    q["m_scale"].copy_(scale8)
    q["m_value"].copy_(torch.where(m < 0, -value, value))
    code, scale8, value = _encode(v, rv, -30)
    q["v"].copy_(code)
    q["v_scale"].copy_(scale8)
    q["v_value"].copy_(value)


def _norm_of(s, to):
    return torch.sqrt(sum(q["grad"].to(to).square().sum() for q in s["sets"].values()))


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "balance":
        return _balance_loss(s, torch.float32)
    if c["kind"] != "adamw":
        r = (_norm_fwd if c["kind"] == "norm_fwd" else _norm_bwd)(s, torch.float32)
        return {k: r[k].to(t.dtype) for k, t in _present(s["out"]).items()}
    s["step"] += 1
    scale = None
    if c["clip"] != "none":
        s["norm_out"][0] = _norm_of(s, torch.float32)
        scale = torch.clamp(s["max_norm"] / (s["norm_out"][0] + 1e-6), max=1.0)
    [_adamw_set(q, s, scale) for q in s["sets"].values()]
    return _adamw_outputs(s, None if scale is None else s["norm_out"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    """The definition in float64 on the inputs of `prepare`, from products, sums
    and the formulas alone."""
    c = case
    if c["kind"] == "adamw":
        return _exact_adamw(_prepare_adamw(c, seed))
    if c["kind"] == "balance":
        return _exact_balance(_prepare_balance(c, seed))
    s = _prepare_norm(c, seed)
    return _exact_fwd(s) if c["kind"] == "norm_fwd" else _exact_bwd(s)


def _d(t):
    return None if t is None else t.double()


def _exact_fwd(s):
    c = s["case"]
    x, y = _d(s["x"]), _d(s["y"])
    out = {}
    if c["post"] != "none":
        mu = y.mean(1) if c["post"] == "layer" else torch.zeros_like(y[:, 0])
        r = (y.square().mean(1) - mu * mu + 1e-6).rsqrt()
        out["post_stats"] = torch.stack([mu, r], 1)
        if s["row_scale"] is not None:
            out["post_stats"][s["row_scale"] == 0] = 0
        y = (y - mu[:, None]) * r[:, None] * _d(s["post_w"])
        y = y + (0 if s["post_b"] is None else _d(s["post_b"]))
    a = torch.ones_like(x[:, 0]) if s["row_scale"] is None else _d(s["row_scale"])
    gate = torch.ones_like(x[:1]) if s["gate"] is None else _d(s["gate"])
    G = gate.shape[0]
    y = (y.view(G, -1, c["d"]) * gate[:, None] * a.view(G, -1, 1)).view_as(x)
    x = x + y
    mu = x.mean(1) if c["pre"] == "layer" else torch.zeros_like(x[:, 0])
    r = (x.square().mean(1) - mu * mu + 1e-6).rsqrt()
    h = (x - mu[:, None]) * r[:, None] * _d(s["pre_w"])
    h = h + (0 if s["pre_b"] is None else _d(s["pre_b"]))
    return dict(out, x_out=x, h=h, pre_stats=torch.stack([mu, r], 1))


def _exact_bwd(s):
    c, d = s["case"], s["case"]["d"]
    x, y, dh, w = _d(s["x"]), _d(s["y"]), _d(s["dh"]), _d(s["pre_w"])
    mu, r = _d(s["pre_stats"]).unbind(1)
    n = x.sub(mu[:, None]).mul_(r[:, None])
    out = dict(dpre_w=torch.einsum("td,td->d", dh, n))
    if s["pre_b"] is not None:
        out["dpre_b"] = dh.sum(0)
    dn = dh * w
    b = (dn * n).sum(1) / d
    a = dn.sum(1) / d if c["pre"] == "layer" else torch.zeros_like(b)
    dx = _d(s["dx_out"]) + r[:, None] * (dn - a[:, None] - b[:, None] * n)
    out["dx"] = dx
    scaled = dx if s["row_scale"] is None else dx * _d(s["row_scale"])[:, None]
    gate = torch.ones_like(x[:1]) if s["gate"] is None else _d(s["gate"])
    G = gate.shape[0]
    pw = torch.ones_like(x[0]) if s["post_w"] is None else _d(s["post_w"])
    pb = torch.zeros_like(x[0]) if s["post_b"] is None else _d(s["post_b"])
    if c["post"] != "none":
        my, ry = _d(s["post_stats"]).unbind(1)
        y = (y - my[:, None]) * ry[:, None]
    S = (scaled * y).view(G, -1, d).sum(1)
    T = scaled.view(G, -1, d).sum(1)
    if s["gate"] is not None:
        out["dgate"] = S * pw + T * pb
    if s["post_w"] is not None:
        out["dpost_w"] = (S * gate).sum(0)
    if s["post_b"] is not None:
        out["dpost_b"] = (T * gate).sum(0)
    dy = (scaled.view(G, -1, d) * (gate * pw)[:, None]).view_as(x)
    if c["post"] != "none":
        b = (dy * y).sum(1) / d
        a = dy.sum(1) / d if c["post"] == "layer" else torch.zeros_like(b)
        dy = ry[:, None] * (dy - a[:, None] - b[:, None] * y)
    return dict(out, dy=dy)


def _exact_balance(s):
    c = s["case"]
    G, E, k = c["groups"], c["experts"], c["k"]
    z = _d(s["logits"])
    if s["bias"] is not None:
        z = z + _d(s["bias"])
    if s["noise"] is not None:
        z = z + _d(s["noise"])
    lse = torch.logsumexp(z, 1)
    n = z.shape[0]
    group = torch.arange(n, device=DEV) // (n // G)
    live = torch.ones(n, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"] != 0
    flat = (group[:, None] * E + s["expert_idx"])[live].reshape(-1)
    demand = torch.bincount(flat, minlength=G * E).view(G, E)
    count = torch.bincount(group[live], minlength=G).clamp(min=1).double()[:, None]
    p = _d(s["probs"]) * live[:, None]
    f = demand.double() / k / count
    P = p.view(G, -1, E).sum(1) / count
    zl = (lse * lse * live).view(G, -1).sum(1) / count[:, 0]
    p3 = p.view(G, -1, E)
    inner = torch.matmul(p3, f[:, :, None])
    grad = s["w_balance"] * E * p3 * (f[:, None] - inner) + \
        2 * s["w_z"] * lse.view(G, -1, 1) * p3
    return dict(losses=torch.stack([E * (f * P).sum(1), zl], 1), demand=demand.to(torch.int32),
                mean_probs=P, dlogits=(grad / count[:, None]).view(n, E))


def _exact_value(code, bits, scale):
    """What codes of `bits` exponent bits and 3 mantissa bits stand for."""
    e, frac = (code // 8).double(), (code % 8).double() / 8
    top = 2.0 ** bits - 1  # the highest exponent counts from 1 to 2
    u = torch.where(e == 0, frac * 2.0 ** (1 - top), (1 + frac) * 2.0 ** (e - top))
    return u * (2.0 ** (scale.double() - 127)).repeat_interleave(BLOCK)


def _exact_adamw(s):
    """States in 8 bits: the values before they are rounded."""
    c, h, t = s["case"], s["hyper"], s["step"] + 1
    out, coef = {}, 1.0
    if c["clip"] != "none":
        total = math.sqrt(sum(q["grad"].double().pow(2).sum().item() for q in s["sets"].values()))
        coef = min(1.0, s["max_norm"] / (total + 1e-6))
        out["norm"] = torch.tensor([total], dtype=torch.float64)
    for kind, q in s["sets"].items():
        m, v = q["m"].double(), q["v"].double()
        if kind == "8bit":
            m = _exact_value(q["m"] & 127, 4, q["m_scale"])
            m = m * torch.where(q["m"] > 127, -1.0, 1.0)
            v = _exact_value(q["v"], 5, q["v_scale"])
        g = q["grad"].double() * coef
        m = h["beta1"] * m + (1 - h["beta1"]) * g
        v = h["beta2"] * v + (1 - h["beta2"]) * g * g
        update = m / (1 - h["beta1"] ** t) / ((v / (1 - h["beta2"] ** t)).sqrt() + h["eps"])
        p = q["master"].double()
        p = p - h["lr"] * update - h["lr"] * q["decay"].double() * p
        out[kind] = _present(dict(param=p if q["param"] is not None else None, master=p, m=m, v=v))
    return out
