"""Cases of the operators of latent attention: one latent vector per token, shared by all heads, in a paged cache.

A case is one call that a program that serves such a target model with speculative drafts makes once per layer and step:

  append   the step's latents (normalised on the way, or as they are) and rotated shared keys into the cache
  absorb   queries of all heads taken into the latent space by their head's key weights, their rotary part rotated
  attn     attention of all draft tokens and heads over the latents
  expand   results out of the latent space by their head's value weights
  compact  the accepted path of each draft tree moved to consecutive slots

`own` false: elementary torch operations in 32 bits (angles in 64); true: the framework's entry points.  A row of the cache is
latent_dim entries, keys and values at once, and rope_dim entries that only keys have.  Sizes are generic.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16


def _case(name, op, batch, heads, ctx, nodes, **more):
    c = {"op": op, "batch": batch, "heads": heads, "latent": 512, "rope": 64, "nope": 128, "value": 128, "ctx_kind": "fixed",
         "ctx": ctx, "ctx_max": ctx, "tree": "", "nodes_min": nodes, "nodes": nodes, "interleaved": True, "theta": 10000.0,
         "norm": True, "out": "bf16", "lse": False, "mix": 0}
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one request, four drafts: the smallest call, launch and latency are all there is
        _case("append_tiny", "append", 1, 16, 256, 4),
        # prompts of many lengths behind a shared system prompt
        _case("append_prompt", "append", 8, 128, 0, 4001, ctx_kind="uniform", ctx_max=777, nodes_min=501, theta=500000.0),
        # single tokens of a serving batch, all heads: the weights are most of what is read
        _case("absorb_token", "absorb", 64, 128, 2048, 1, ctx_kind="lognormal", ctx_max=16384),
        # draft trees: queries of 64 nodes each, halves rotated
        _case("absorb_tree", "absorb", 16, 128, 4096, 64, tree="4,4,2,2", interleaved=False),
        # the smallest attention call
        _case("attn_tiny", "attn", 1, 16, 256, 4),
        # single tokens, an eighth of the heads (the others on other devices), ragged contexts: bound by memory
        _case("attn_token", "attn", 64, 16, 2048, 1, ctx_kind="lognormal", ctx_max=16384),
        # the serving batch with all heads: ragged contexts and drafts, the most matrix work
        _case("attn_serving", "attn", 64, 128, 2048, 10, ctx_kind="lognormal", ctx_max=16384, nodes_min=2),
        # draft trees of a smaller model, odd lengths, results and log-sum-exp in fp32
        _case("attn_tree", "attn", 5, 40, 1001, 61, latent=256, rope=32, nope=64, value=64, ctx_kind="uniform", ctx_max=7999,
              tree="4,4,2,2", out="f32", lse=True),
        # results of the serving batch
        _case("expand_serving", "expand", 64, 128, 2048, 10, nodes_min=2),
        # ... of one request, an eighth of the heads
        _case("expand_small", "expand", 1, 16, 256, 7),
        # accepted paths of full trees
        _case("compact_tree", "compact", 16, 128, 4096, 116, tree="4,4,2,2"),
        # ... of small ones, a smaller model
        _case("compact_small", "compact", 3, 40, 333, 21, latent=256, rope=32, ctx_kind="uniform", ctx_max=999, tree="3,2,2"),
    ]


def _between(rng, lo, hi):
    """A whole number whose logarithm is uniform between those of lo and hi."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "absorb", "absorb", "attn", "attn", "attn", "attn", "expand", "expand", "compact"])
    while True:
        c = _case("", op, _between(rng, 1, 64), rng.choice([1, 5, 8, 16, 16, 20, 32, 40, 64, 128]), _between(rng, 16, 16384),
                  rng.randint(1, 16), mix=rng.randrange(1 << 20))
        c["latent"], c["rope"] = rng.choice([(512, 64), (512, 64), (512, 32), (256, 64), (256, 32)])
        c["nope"], c["value"] = rng.choice([64, 128, 128]), rng.choice([64, 128, 128])
        c["ctx_kind"] = rng.choice(["fixed", "uniform", "lognormal"])
        c["ctx_max"] = c["ctx"] if c["ctx_kind"] == "fixed" else min(16384, c["ctx"] * rng.randint(2, 6))
        if op == "append" and rng.random() < 0.4:                           # prompts
            c["ctx_kind"], c["ctx"], c["ctx_max"] = "uniform", 0, rng.randint(1, 2000)
            c["nodes"] = _between(rng, 100, 8000)
        c["nodes_min"] = rng.randint(1, c["nodes"])
        if op == "compact" or (c["nodes"] <= 16 and rng.random() < 0.4):
            c["tree"], c["nodes"] = rng.choice([("4,4,2,2", rng.randint(20, 116)), ("2,2,2,2", rng.randint(8, 30)),
                                                ("3,2,2", rng.randint(6, 21)), ("8,4,2", rng.randint(16, 104))])
            c["nodes_min"] = c["nodes"]
        c["interleaved"] = rng.random() < 0.6
        c["norm"] = rng.random() < 0.7
        c["theta"] = rng.choice([10000.0, 500000.0, 1000000.0])
        if op == "attn":
            c["lse"] = rng.random() < 0.3
            c["out"] = rng.choice(["bf16", "bf16", "bf16", "f32"])
        w = work(c)
        ctx, n, _, _ = _structure(c)
        held = 4.0 * int((ctx + n).max()) * c["batch"] * (c["latent"] + c["rope"] + c["heads"] * int(n.max()))
        if w["bytes"] < 4e8 and w["flops"] < 3e11 and (op != "attn" or held < 8e9):
            return c


# ----------------------------------------------------------------------------------------------------------------
# sizes of a case: its own, whatever the seed
# ----------------------------------------------------------------------------------------------------------------
def _tree(branching, most):
    """Parents of the full tree with that branching by depth, breadth first, its first `most` nodes."""
    parents, level = np.array([], dtype=np.int64), np.array([-1])
    for br in branching:
        level, parents = len(parents) + np.arange(len(level) * br), np.concatenate([parents, np.repeat(level, br)])
    return parents[:most]


def _structure(c):
    """(context lengths, new tokens per request, parents within one request or None, last accepted node per request)."""
    r = np.random.RandomState(c["mix"])
    B = c["batch"]
    if c["ctx_kind"] == "fixed":
        ctx = np.full(B, c["ctx"])
    elif c["ctx_kind"] == "uniform":
        ctx = r.randint(c["ctx"], c["ctx_max"] + 1, B)
    else:
        ctx = np.clip(np.rint(c["ctx"] * np.exp(0.8 * r.standard_normal(B))), min(512, c["ctx"]), c["ctx_max"])
    parent = _tree([int(x) for x in c["tree"].split(",")], c["nodes"]) if c["tree"] else None
    n = np.full(B, len(parent)) if parent is not None else r.randint(c["nodes_min"], c["nodes"] + 1, B)
    stop = r.randint(-1, n)
    return ctx.astype(np.int64), n.astype(np.int64), parent, stop.astype(np.int64)


def work(case):
    c = case
    ctx, n, parent, stop = _structure(c)
    C, R, H, total = c["latent"], c["rope"], c["heads"], int(n.sum())
    W = C + R
    if c["op"] == "append":
        return {"bytes": float(4 * total * W + 2 * C * c["norm"]), "flops": float(total * (4 * C * c["norm"] + 3 * R))}
    if c["op"] == "absorb":
        return {"bytes": float(2 * total * H * (c["nope"] + R + W) + 2 * H * c["nope"] * C), "flops": float(2 * total * H * c["nope"] * C)}
    if c["op"] == "expand":
        return {"bytes": float(2 * total * H * (C + c["value"]) + 2 * H * c["value"] * C), "flops": float(2 * total * H * c["value"] * C)}
    if c["op"] == "compact":
        path = 0
        for s in stop.tolist():
            while s >= 0:
                s, path = int(parent[s]), path + 1
        return {"bytes": float(4 * path * W + 12 * c["batch"]), "flops": float(path * W)}
    L = ctx + n
    by = 2 * W * L + n * H * (2 * W + C * (4 if c["out"] == "f32" else 2) + 4 * c["lse"])
    return {"bytes": float(by.sum()), "flops": float((2 * n * H * L * (W + C)).sum())}


# ----------------------------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------------------------
def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


class _State:
    pass


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ctx, n, parent, stop = _structure(c)
    B, H, C, R, N, V, total = c["batch"], c["heads"], c["latent"], c["rope"], c["nope"], c["value"], int(n.sum())
    W = C + R
    s = _State()
    s.op, s.C, s.N, s.total, s.interleaved = c["op"], C, N, total, c["interleaved"]
    s.scale = (N + R) ** -0.5
    pages = (ctx + n + PAGE - 1) // PAGE
    held = int(pages.sum()) + 3
    perm = np.random.RandomState(seed % (1 << 32)).permutation(held)
    table = np.full((B, int(pages.max())), -1)
    at = 0
    for b in range(B):
        table[b, :pages[b]] = perm[at:at + pages[b]]
        at += int(pages[b])
    s.table, s.ctx, s.stop = _i32(table), _i32(ctx), _i32(stop)
    s.offsets = _i32(np.concatenate([[0], np.cumsum(n)]))
    s.parent = None if parent is None else _i32(np.tile(parent, B))
    s.most, s.longest = int(n.max()), int((ctx + n).max())
    s.new_len = torch.empty(B, dtype=torch.int32, device="cuda")

    def normal(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=g)

    s.inv_freq = (c["theta"] ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)).float().cuda()
    if s.op in ("append", "attn", "compact"):
        s.pool = normal(held, PAGE, W)
    if s.op == "append":                # as one projection leaves them
        x = torch.randn((total, W), generator=g, device="cuda") * torch.exp2(2 * torch.rand((total, 1), generator=g, device="cuda") - 1)
        s.latent, s.key = x.bfloat16().split((C, R), 1)
        s.norm = (1 + 0.1 * torch.randn(C, generator=g, device="cuda")).bfloat16() if c["norm"] else None
    if s.op in ("absorb", "expand"):    # the two halves of one weight
        w = torch.randn((H, N + V, C), generator=g, device="cuda")
        w[:, :N] *= N ** -0.5
        w[:, N:] *= C ** -0.5
        s.w_key, s.w_value = w.bfloat16().split((N, V), 1)
    if s.op == "absorb":
        s.q = normal(total, H, N + R)
        s.out = torch.empty((total, H, W), dtype=torch.bfloat16, device="cuda")
    if s.op == "expand":
        s.x = normal(total, H, C)
        s.out = torch.empty((total, H, V), dtype=torch.bfloat16, device="cuda")
    if s.op == "attn":                  # heads that look at few tokens, and at many
        s.q = (torch.randn((total, H, W), generator=g, device="cuda")
               * torch.exp2(2 * torch.rand((1, H, 1), generator=g, device="cuda") - 1)).bfloat16()
        s.out = torch.empty((total, H, C), dtype=torch.float32 if c["out"] == "f32" else torch.bfloat16, device="cuda")
        s.lse = torch.empty((total, H), dtype=torch.float32, device="cuda") if c["lse"] else None
    if own:
        from paper_2503_10325_amd import binding as sv
        s.sv = sv
        s.desc = sv.make_latent_desc(B, H, C, R, N, V, total, s.most, table.shape[1], held, interleaved=c["interleaved"], norm_eps=1e-6,
                                     out_dtype=sv.SPEC_F32 if c["out"] == "f32" else sv.SPEC_BF16)
        if s.op == "attn":
            s.workspace = torch.empty(max(256, sv.spec_verify_attn_latent_workspace_size(s.desc)), dtype=torch.uint8, device="cuda")
    return s


# ----------------------------------------------------------------------------------------------------------------
# plain forms
# ----------------------------------------------------------------------------------------------------------------
def _places(s):
    """(request, index within the request) of every new token."""
    t = torch.arange(s.total, device="cuda")
    b = torch.searchsorted(s.offsets[1:].long(), t, right=True)
    return b, t - s.offsets[b]


def _lineage(s, b, i):
    """[requests, nodes, nodes]: whether the second node is the first or an ancestor of it."""
    B, m = s.ctx.shape[0], s.most
    if s.parent is None:
        return torch.ones((m, m), dtype=torch.bool, device="cuda").tril().expand(B, m, m)
    step = torch.eye(m, device="cuda").repeat(B, 1, 1)
    has = s.parent >= 0
    step[b[has], i[has], s.parent[has].long()] = 1.0
    return torch.linalg.matrix_power(step, 128) > 0            # chains of up to 128 nodes: binomials below 2.4e37


def _rotated(s, x, b, i):
    """x [tokens, heads, R] in 32 bits, rotated by its positions."""
    depth = i if s.parent is None else _lineage(s, b, i).sum(-1)[b, i] - 1
    a = (s.ctx[b] + depth).double()[:, None] * s.inv_freq.double()
    cos, sin = a.cos().float()[:, None], a.sin().float()[:, None]
    x = x.float()
    if s.interleaved:
        u, w = x[..., 0::2], x[..., 1::2]
        return torch.stack((u * cos - w * sin, w * cos + u * sin), -1).flatten(-2)
    u, w = x.chunk(2, -1)
    return torch.cat((u * cos - w * sin, w * cos + u * sin), -1)


def _append_plain(s):
    b, i = _places(s)
    at = s.ctx[b] + i
    page, slot = s.table[b, at // PAGE].long(), (at % PAGE).long()
    z = s.latent.float()
    if s.norm is not None:
        z = z * torch.rsqrt((z * z).mean(-1, keepdim=True) + 1e-6) * s.norm.float()
    s.pool[page, slot] = torch.cat((z, _rotated(s, s.key[:, None], b, i)[:, 0]), -1).bfloat16()
    return {"pool": s.pool}


def _absorb_plain(s):
    b, i = _places(s)
    nope, rope = s.q[..., :s.N], s.q[..., s.N:]
    z = torch.matmul(nope.float().transpose(0, 1).contiguous(), s.w_key.float()).transpose(0, 1)
    return {"q": torch.cat((z, _rotated(s, rope, b, i)), -1).bfloat16()}


def _expand_plain(s):
    w = s.w_value.float().transpose(1, 2).contiguous()
    return {"out": torch.matmul(s.x.float().transpose(0, 1).contiguous(), w).transpose(0, 1).bfloat16()}


def _attn_plain(s):
    b, i = _places(s)
    B, m, P = s.ctx.shape[0], s.most, s.table.shape[1]
    H, W = s.q.shape[1:]
    rows = s.pool[s.table.long().clamp(min=0)].float().view(B, P * PAGE, W)
    q = torch.zeros((B, m, H, W), device="cuda")
    q[b, i] = s.q.float()
    t = torch.arange(P * PAGE, device="cuda")[None] - s.ctx[:, None]                  # place behind the context
    mask = _lineage(s, b, i).gather(2, t.clamp(0, m - 1)[:, None].expand(B, m, -1).long())
    mask = (t < 0)[:, None] | (mask & (t < (s.offsets[1:] - s.offsets[:-1])[:, None])[:, None])
    x = torch.matmul(q.view(B, m * H, W), rows.transpose(1, 2).contiguous()).mul_(s.scale).view(B, m, H, -1)
    x.masked_fill_(~mask[:, :, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)            # rows that are padding see nothing
    x = (x - top).exp_()
    z = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, m * H, -1), rows[..., :s.C].contiguous()).view(B, m, H, -1) / z
    got = {"out": o[b, i].to(s.out.dtype)}
    if s.lse is not None:
        got["lse"] = (top + z.log())[b, i][..., 0]
    return got


def _compact_plain(s):
    b, i = _places(s)
    kin = _lineage(s, b, i)
    on = kin[b, s.stop[b].long().clamp(min=0), i] & (s.stop[b] >= 0)
    to = (kin.sum(-1)[b, i] - 1)[on]
    b, i = b[on], i[on]
    frm, to = s.ctx[b] + i, s.ctx[b] + to
    moved = s.pool[s.table[b, frm // PAGE].long(), (frm % PAGE).long()]
    s.pool[s.table[b, to // PAGE].long(), (to % PAGE).long()] = moved
    new_len = s.ctx + torch.zeros_like(s.ctx).index_add_(0, b, torch.ones_like(b, dtype=torch.int32))
    return {"pool": s.pool, "new_len": new_len}


def run(state):
    s = state
    if not own:
        return {"append": _append_plain, "absorb": _absorb_plain, "attn": _attn_plain, "expand": _expand_plain,
                "compact": _compact_plain}[s.op](s)
    if s.op == "append":
        s.sv.spec_append_latent(s.desc, s.latent, s.key, s.norm, s.inv_freq, s.pool, s.table, s.ctx, s.offsets, s.parent)
        return {"pool": s.pool}
    if s.op == "absorb":
        s.sv.spec_absorb_latent(s.desc, s.q, s.w_key, s.inv_freq, s.ctx, s.offsets, s.parent, s.out)
        return {"q": s.out}
    if s.op == "attn":
        s.sv.spec_verify_attn_latent(s.desc, s.q, s.pool, s.table, s.ctx, s.offsets, s.parent, s.out, s.lse, s.workspace)
        return {"out": s.out} if s.lse is None else {"out": s.out, "lse": s.lse}
    if s.op == "expand":
        s.sv.spec_expand_latent(s.desc, s.x, s.w_value, s.offsets, s.out)
        return {"out": s.out}
    s.sv.spec_compact_latent(s.pool, s.table, s.ctx, s.offsets, s.parent, s.stop, s.new_len)
    return {"pool": s.pool, "new_len": s.new_len}


# ----------------------------------------------------------------------------------------------------------------
# from the definition, in 64 bits, request by request
# ----------------------------------------------------------------------------------------------------------------
def _chain(parent, j):
    """Node j and its ancestors, from the root."""
    up = []
    while j >= 0:
        up.append(j)
        j = int(parent[j]) if parent is not None else j - 1
    return up[::-1]


def _turned(x, pos, inv_freq, interleaved):
    x = x.double()
    h = inv_freq.shape[0]
    unit = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos.double()[:, None] * inv_freq.double())
    unit = unit.view(-1, *([1] * (x.dim() - 2)), h)
    first, second = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if interleaved else (slice(0, h), slice(h, 2 * h))
    z = torch.complex(x[..., first], x[..., second]) * unit
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    ctx, n, parent, stop = _structure(c)
    if c["op"] == "expand":
        return {"out": torch.stack([torch.matmul(s.x[:, h].double(), s.w_value[h].double().t().contiguous()) for h in range(c["heads"])], 1)}
    first = s.offsets.tolist()
    pool = s.pool.double() if c["op"] in ("append", "compact") else None
    got, got_l = [], []
    for b in range(c["batch"]):
        L, m = int(ctx[b]), int(n[b])
        rows = slice(first[b], first[b] + m)
        chains = None if parent is None else [_chain(parent, j) for j in range(m)]
        depth = torch.arange(m, device="cuda") if chains is None else torch.tensor([len(x) - 1 for x in chains], device="cuda")
        at = L + torch.arange(m, device="cuda")
        if c["op"] == "append":
            z = s.latent[rows].double()
            if s.norm is not None:
                z = z / ((z ** 2).sum(-1, keepdim=True) / s.C + 1e-6).sqrt() * s.norm.double()
            k = _turned(s.key[rows], L + depth, s.inv_freq, c["interleaved"])
            pool[s.table[b][at // PAGE].long(), at % PAGE] = torch.cat((z, k), 1)
        elif c["op"] == "absorb":
            q = s.q[rows].double()
            z = torch.stack([torch.matmul(q[:, h, :s.N].contiguous(), s.w_key[h].double()) for h in range(c["heads"])], 1)
            got.append(torch.cat((z, _turned(q[..., s.N:], L + depth, s.inv_freq, c["interleaved"])), -1))
        elif c["op"] == "compact":
            path = torch.tensor([] if stop[b] < 0 else _chain(parent, int(stop[b])), dtype=torch.long, device="cuda")
            to = L + torch.arange(len(path), device="cuda")
            moved = pool[s.table[b][(L + path) // PAGE].long(), (L + path) % PAGE].clone()
            pool[s.table[b][to // PAGE].long(), to % PAGE] = moved
        else:
            kv = s.pool[s.table[b][:(L + m + PAGE - 1) // PAGE].long()].double().view(-1, s.pool.shape[2])[:L + m]
            sees = torch.ones((m, L + m), dtype=torch.bool, device="cuda")
            if chains is None:
                sees[:, L:] = torch.ones((m, m), dtype=torch.bool).tril().cuda()
            else:
                kin = torch.zeros((m, m), dtype=torch.bool)
                for j, up in enumerate(chains):
                    kin[j, up] = True
                sees[:, L:] = kin.cuda()
            keys, values = kv.t().contiguous(), kv[:, :s.C].contiguous()
            for j in range(m):
                x = (torch.matmul(s.q[first[b] + j].double(), keys) * (c["nope"] + c["rope"]) ** -0.5).masked_fill(~sees[j], -math.inf)
                l = torch.logsumexp(x, -1)
                got.append(torch.matmul((x - l[:, None]).exp(), values)[None])
                got_l.append(l[None])
    if c["op"] == "append":
        return {"pool": pool}
    if c["op"] == "compact":
        return {"pool": pool, "new_len": None}
    if c["op"] == "absorb":
        return {"q": torch.cat(got)}
    return {"out": torch.cat(got)} if s.lse is None else {"out": torch.cat(got), "lse": torch.cat(got_l)}
