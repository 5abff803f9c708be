"""Inputs of the cache operators' tests: a batch as a dict of host arrays, and its device copies."""
import numpy as np

from oracle import cache as R
from paper_2503_10325_amd import workloads as W


def bf16(x):
    """Rounded to bf16, as float32."""
    return W.bf16_bits_to_f32(W.f32_to_bf16_bits(np.asarray(x, dtype=np.float32)))


def random_tree(rng, n):
    return np.array([rng.integers(-1, i) if i else -1 for i in range(n)], dtype=np.int32)


def batch(seed, ctx, n, heads=(4, 2), D=128, tree=False, rotary=None, interleaved=False, scale=1.0, theta=10000.0, spare=3,
          positions=None, rows_behind=0):
    """q, k, v, offsets, table and so on of a batch with those context lengths and new tokens."""
    rng = np.random.default_rng(seed)
    ctx, n = np.asarray(ctx, dtype=np.int32), np.asarray(n, dtype=np.int32)
    Hq, Hkv = heads
    offsets = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    total = int(offsets[-1])
    pages = (ctx.astype(np.int64) + n + R.PAGE - 1) // R.PAGE
    held = int(pages.sum()) + spare
    perm = rng.permutation(held)
    table = np.full((len(ctx), max(1, int(pages.max(initial=1)))), -1, dtype=np.int32)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = perm[at:at + p]
        at += int(p)
    rotary = D if rotary is None else rotary
    rows = total + rows_behind
    c = dict(ctx=ctx, n=n, offsets=offsets, total=total, rows=rows, table=table, held=held, heads=heads, D=D, rotary=rotary,
             interleaved=interleaved, scale=scale, positions=positions, rng=rng,
             parent=np.concatenate([random_tree(rng, int(m)) for m in n] or [[]]).astype(np.int32) if tree else None,
             inv_freq=(theta ** (-np.arange(0, rotary, 2) / max(rotary, 1))).astype(np.float32) if rotary else None)
    if rows_behind and c["parent"] is not None:
        c["parent"] = np.concatenate([c["parent"], np.full(rows_behind, -1, dtype=np.int32)])
    for name, h in (("q", Hq), ("k", Hkv), ("v", Hkv)):
        c[name] = bf16(rng.standard_normal((rows, h, D)) * 2.0 ** rng.uniform(-1, 1, (rows, h, 1)))
    return c


def quant_pools(c, spread=2):
    """Pools of random codes (no NaN) and power-of-two scales."""
    rng, (_, H), D = c["rng"], c["heads"], c["D"]
    code = lambda shape: ((rng.integers(0, 2, shape) << 7) | rng.integers(0, 0x7f, shape)).astype(np.uint8)
    # codes near 1 to 16, as entries ~ N(0, 1) against a scale of their largest have, and some of any size
    def some(shape):
        x = R.encode_e4m3(np.clip(rng.standard_normal(shape) * 100, -448, 448))
        return np.where(rng.random(shape) < 0.02, code(shape), x).astype(np.uint8)
    scales = lambda: (2.0 ** rng.integers(-7 - spread, -7 + spread + 1, (c["held"], H))).astype(np.float32)
    return some((c["held"], H, D // 16, 16, 16)), some((c["held"], H, D, 16)), scales(), scales()


class Device:
    """Device copies of a batch and calls of the operators on them."""

    def __init__(self, c, fused=False, quant=None, bf16_pools=None, device="cuda"):
        import torch

        from paper_2503_10325_amd import binding as sv
        self.sv, self.torch, self.c = sv, torch, c
        dev = lambda x, t=None: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(device, t)
        b16 = lambda x: dev(x, torch.bfloat16)
        Hq, Hkv = c["heads"]
        if fused:
            qkv = b16(np.concatenate([c["q"], c["k"], c["v"]], axis=1))
            self.q, self.k, self.v = qkv.split((Hq, Hkv, Hkv), 1)
        else:
            self.q, self.k, self.v = b16(c["q"]), b16(c["k"]), b16(c["v"])
        self.inv_freq, self.positions = dev(c["inv_freq"]), dev(c["positions"])
        self.table, self.ctx, self.offsets, self.parent = dev(c["table"]), dev(c["ctx"]), dev(c["offsets"]), dev(c["parent"])
        self.q_out = torch.full((c["rows"], Hq, c["D"]), 7.0, dtype=torch.bfloat16, device=device)
        most = int(c["n"].max(initial=0))
        self.append_desc = sv.make_append_desc(len(c["ctx"]), Hq, Hkv, c["D"], c["rows"], most, c["table"].shape[1], c["held"],
                                               c["rotary"], c["interleaved"], 0.0 if c["scale"] == 1.0 else c["scale"])
        if quant is not None:
            self.k_pool, self.v_pool, self.k_scale, self.v_scale = (dev(x) for x in quant)
        if bf16_pools is not None:
            self.k_pool, self.v_pool = (b16(x) for x in bf16_pools)

    def append(self, q="given", stream=None, q_out="own"):
        q = self.q if isinstance(q, str) else q
        out = self.q_out if isinstance(q_out, str) else q_out
        pools = (self.k_pool, self.v_pool)
        if hasattr(self, "k_scale"):
            self.sv.spec_append_kv_quant(self.append_desc, q, self.k, self.v, self.inv_freq, *pools, self.k_scale, self.v_scale,
                                         self.table, self.ctx, self.offsets, self.parent, out, self.positions, stream)
        else:
            self.sv.spec_append_kv(self.append_desc, q, self.k, self.v, self.inv_freq, *pools, self.table, self.ctx, self.offsets,
                                   self.parent, out, self.positions, stream)

    def attend(self, q, f32=False, lse=True, stream=None, scale=0.0):
        torch, c = self.torch, self.c
        if not hasattr(self, "attn_desc") or self.attn_desc.out_dtype != int(f32):
            self.attn_desc = self.sv.make_attn_desc(len(c["ctx"]), *c["heads"], c["D"], q.shape[0], int(c["n"].max(initial=0)),
                                                    c["table"].shape[1], 0, scale, self.sv.SPEC_F32 if f32 else self.sv.SPEC_BF16)
            # (as a caller's memory may be: full of NaN)
            self.workspace = torch.full((max(256, self.sv.spec_verify_attn_quant_workspace_size(self.attn_desc)),), 0xff,
                                        dtype=torch.uint8, device="cuda")
            self.out = torch.full(q.shape, 7.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
            self.lse = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device="cuda") if lse else None
        self.sv.spec_verify_attn_quant(self.attn_desc, q, self.k_pool, self.v_pool, self.k_scale, self.v_scale, self.table, self.ctx,
                                       self.offsets, self.parent, self.out, self.lse, self.workspace, stream)
        return self.out, self.lse

    def compact(self, stop, stream=None):
        new_len = self.torch.full((len(self.c["ctx"]),), -5, dtype=self.torch.int32, device="cuda")
        self.sv.spec_compact_kv_quant(self.k_pool, self.v_pool, self.k_scale, self.v_scale, self.table, self.ctx, self.offsets,
                                      self.parent, stop, new_len, stream)
        return new_len


def host(t):
    return t.detach().float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


# ---- comparisons, by the arithmetic of the roundings ----
def rotated_close(got, true, x, rotary, rounding):
    """got: rounded results, true: 64-bit ones, x: the inputs.  A rotated value is off by its own rounding (half a step, `rounding`
    relative) and by fp32 arithmetic on its pair: cosine and sine to 2^-22, two products and a sum at 2^-24 each, of at most
    |x1| + |x2|: 2^-21 of it, the pair bounded by twice the head's largest."""
    slack = 2.0 ** -20 * np.abs(x).max(-1, keepdims=True) if rotary else 0.0
    return np.all(np.abs(got - true) <= np.abs(true) * rounding + slack)


def attn_close(got, ref, v_abs, f32):
    """out = sum p v: each weight is off by 2^-11 (one fp16 term, rounding of the exponential's argument included) or 2^-18 (two
    terms; scores up to 2^5 in fp32: 2^5 2^-24 log2(e) twice), relative, of sum p |v| <= the largest |v|; plus the result's own
    rounding: bf16 2^-8, fp32 2^-24."""
    own, weight = (2.0 ** -24, 2.0 ** -16) if f32 else (2.0 ** -8, 2.0 ** -10)
    return np.all(np.abs(got - ref) <= own * np.abs(ref) + weight * v_abs)
