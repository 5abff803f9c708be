"""Inputs of the latent operators' tests: a batch as a dict of host arrays, and its device copies and calls."""
import numpy as np

from cache_util import bf16, random_tree
from oracle import cache as R

EPS = 1e-6


def batch(seed, ctx, n, H=4, C=512, rope=64, nope=128, value=128, tree=False, interleaved=False, scale=1.0, theta=10000.0, spare=3, positions=None,
          rows_behind=0, spread=1.0):
    """offsets, table, the step's tensors, weights and the pool of a batch with those context lengths and new tokens."""
    rng = np.random.default_rng(seed)
    ctx, n = np.asarray(ctx, dtype=np.int32), np.asarray(n, dtype=np.int32)
    offsets = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    total = int(offsets[-1])
    rows = total + rows_behind
    pages = (np.maximum(ctx, 0).astype(np.int64) + n + R.PAGE - 1) // R.PAGE
    held = int(pages.sum()) + spare
    perm = rng.permutation(held)
    table = np.full((len(ctx), max(1, int(pages.max(initial=1)))), -1, dtype=np.int32)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = perm[at:at + p]
        at += int(p)
    W = C + rope
    c = dict(ctx=ctx, n=n, offsets=offsets, total=total, rows=rows, table=table, held=held, H=H, C=C, rope=rope, nope=nope, value=value,
             interleaved=interleaved, scale=scale, positions=positions, rng=rng,
             parent=np.concatenate([random_tree(rng, int(m)) for m in n] or [[]]).astype(np.int32) if tree else None,
             inv_freq=(theta ** (-np.arange(0, rope, 2) / rope)).astype(np.float32))
    if rows_behind and c["parent"] is not None:
        c["parent"] = np.concatenate([c["parent"], np.full(rows_behind, -1, dtype=np.int32)])
    some = lambda *shape: bf16(rng.standard_normal(shape) * 2.0 ** rng.uniform(-spread, spread, shape[:-1] + (1,)))
    c.update(latent=some(rows, C), key=some(rows, rope), q=some(rows, H, nope + rope), ql=some(rows, H, W), x=some(rows, H, C), pool=some(held, R.PAGE, W),
             norm=bf16(1 + 0.1 * rng.standard_normal(C)),
             w=bf16(np.concatenate([rng.standard_normal((H, nope, C)) * nope ** -0.5, rng.standard_normal((H, value, C)) * C ** -0.5], 1)))
    c["w_key"], c["w_value"] = c["w"][:, :nope], c["w"][:, nope:]
    c["softmax"] = (nope + rope) ** -0.5
    return c


class Device:
    """Device copies of a batch and calls of the operators on them; results start as 7."""

    def __init__(self, c, apart=True, f32=False, softmax=0.0):
        import torch

        from paper_2503_10325_amd import binding as sv
        self.sv, self.torch, self.c = sv, torch, c
        dev = lambda x, t=None: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to("cuda", t)
        b16 = lambda x: dev(x, torch.bfloat16)
        H, C, N = c["H"], c["C"], c["nope"]
        if apart:                       # slices of one projection, of one weight
            self.latent, self.key = b16(np.concatenate([c["latent"], c["key"]], 1)).split((C, c["rope"]), 1)
            self.w_key, self.w_value = b16(c["w"]).split((N, c["value"]), 1)
            self.q = b16(np.concatenate([c["q"], c["q"][:, :1]], 1))[:, :H]
        else:
            self.latent, self.key, self.w_key, self.w_value, self.q = (b16(c[k]) for k in ("latent", "key", "w_key", "w_value", "q"))
        self.norm, self.ql, self.x, self.pool = (b16(c[k]) for k in ("norm", "ql", "x", "pool"))
        self.inv_freq, self.positions = dev(c["inv_freq"]), dev(c["positions"])
        self.table, self.ctx, self.offsets, self.parent = dev(c["table"]), dev(c["ctx"]), dev(c["offsets"]), dev(c["parent"])
        self.desc = sv.make_latent_desc(len(c["ctx"]), H, C, c["rope"], N, c["value"], c["rows"], max(1, int(c["n"].max(initial=0))), c["table"].shape[1], c["held"],
                                        c["interleaved"], 0.0 if c["scale"] == 1.0 else c["scale"], EPS, softmax, sv.SPEC_F32 if f32 else sv.SPEC_BF16)
        sevens = lambda *shape, t=torch.bfloat16: torch.full(shape, 7.0, dtype=t, device="cuda")
        self.q_out, self.out = sevens(c["rows"], H, C + c["rope"]), sevens(c["rows"], H, c["value"])
        self.o, self.lse = sevens(c["rows"], H, C, t=torch.float32 if f32 else torch.bfloat16), sevens(c["rows"], H, t=torch.float32)
        # (as a caller's memory may be: full of NaN)
        self.workspace = torch.full((max(256, sv.spec_verify_attn_latent_workspace_size(self.desc)),), 0xff, dtype=torch.uint8, device="cuda")

    def append(self, norm=True, stream=None):
        self.sv.spec_append_latent(self.desc, self.latent, self.key, self.norm if norm else None, self.inv_freq, self.pool, self.table, self.ctx,
                                   self.offsets, self.parent, self.positions, stream)
        return self.pool

    def absorb(self, stream=None):
        self.sv.spec_absorb_latent(self.desc, self.q, self.w_key, self.inv_freq, self.ctx, self.offsets, self.parent, self.q_out, self.positions, stream)
        return self.q_out

    def attend(self, ql=None, lse=True, stream=None, workspace=None):
        self.sv.spec_verify_attn_latent(self.desc, self.ql if ql is None else ql, self.pool, self.table, self.ctx, self.offsets, self.parent, self.o,
                                        self.lse if lse else None, self.workspace if workspace is None else workspace, stream)
        return self.o, self.lse

    def expand(self, x=None, stream=None):
        self.sv.spec_expand_latent(self.desc, self.x if x is None else x, self.w_value, self.offsets, self.out, stream)
        return self.out

    def compact(self, stop, stream=None):
        new_len = self.torch.full((len(self.c["ctx"]),), -5, dtype=self.torch.int32, device="cuda")
        self.sv.spec_compact_latent(self.pool, self.table, self.ctx, self.offsets, self.parent, stop, new_len, stream)
        return new_len


def host(t):
    return t.detach().float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


# ---- comparisons, by the arithmetic of the roundings ----
HALF = 2.0 ** -8                        # half a step of bf16, relative


def rotated_close(got, true, x):
    """A rotated value is off by its own rounding and by fp32 arithmetic on its pair: cosine and sine to 2^-22, two products and a sum at 2^-24 each, of
    at most |x1| + |x2|: 2^-21 of it, the pair bounded by twice the row's largest."""
    return np.all(np.abs(got - true) <= HALF * np.abs(true) + 2.0 ** -20 * np.abs(x).max(-1, keepdims=True))


def product_close(got, true, size, K):
    """A sum of K exact products in fp32, rounded once: at most K roundings of 2^-24 of the sum of absolute products (`size`)."""
    return np.all(np.abs(got - true) <= HALF * np.abs(true) + 1.01 * K * 2.0 ** -24 * size)
