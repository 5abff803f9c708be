"""Attention over the 8-bit cache is as accurate as its header says, row by row.

For a row that sees L positions with weights w, A the largest scale * sum_i |q_i k_i| among them, V 448 times the largest scale of v of the request:

    |out - exact| <= (t + e) sum w |v| + 2^-31 L V  (+ half a step of the result's type),   |lse - exact| <= e + 2^-22 |lse|,
    e = 2^-20 (1 + A) + 2^-24 sqrt(L),   t = 2^-11 for bf16 results, 0 for fp32 ones.

t is half a step of a weight in fp16 (a second term takes it to 2^-22, which e holds).  Of e: a score is a sum of D exact products, rounded to fp32 after every
few of them, 2^-24 of at most A each time, some tens of times in either direction, then multiplied and subtracted (2^-24 A each): 2^-21 A for the weight and
for the sum of weights; the exponential 2^-23; sums over L / 32 steps, 2^-24 each, in either direction.  Weights below 2^-20 of the largest are
subnormal in fp16, 2^-31 off at most.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import cache_util as U
from oracle import cache as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_10325_amd import binding
    binding.lib()


def terms(c, pools):
    """A and L of every row and head, V of every (row, head)."""
    k_pool, _, k_scale, v_scale = pools
    G, Hkv, D = c["heads"][0] // c["heads"][1], c["heads"][1], c["D"]
    A, L, V = (np.zeros((c["total"], c["heads"][0])) for _ in range(3))
    for b in range(len(c["ctx"])):
        o, n, ctx = int(c["offsets"][b]), int(c["n"][b]), int(c["ctx"][b])
        if n == 0:
            continue
        at = np.arange(ctx + n)
        page = c["table"][b, at // R.PAGE]
        k = np.abs(R.E4M3[k_pool[page, :, :, at % R.PAGE]].reshape(ctx + n, Hkv, D) * k_scale[page][..., None])
        top = 448.0 * v_scale[page].max(0)
        up = R.chains(None if c["parent"] is None else c["parent"][o:o + n], n)
        q = np.abs(c["q"][o:o + n]).astype(np.float64).reshape(n, Hkv, G, D)
        s = np.einsum("nhgd,thd->nhgt", q, k) / np.sqrt(D)
        for j in range(n):
            sees = np.concatenate([np.ones(ctx, dtype=bool), np.isin(np.arange(n), up[j])])
            A[o + j] = s[j][..., sees].max(-1).reshape(-1)
            L[o + j] = sees.sum()
        V[o:o + n] = np.repeat(top, G)
    return A, L, V


def ratio(c, pools, f32):
    """The largest error by its bound, of results and of log-sum-exp."""
    d = U.Device(c, quant=pools)
    out, lse = d.attend(d.q, f32)
    torch.cuda.synchronize()
    ref, ref_lse = R.attend(c, c["q"], *pools)
    size, _ = R.attend(c, c["q"], pools[0], pools[1] & 0x7f, *pools[2:])          # sum w |v|
    A, L, V = terms(c, pools)
    e = 2.0 ** -20 * (1 + A) + 2.0 ** -24 * np.sqrt(L)
    own, t = (2.0 ** -24, 0.0) if f32 else (2.0 ** -8, 2.0 ** -11)
    bound = (t + e)[..., None] * size + (2.0 ** -31 * L * V)[..., None]
    got = np.abs(U.host(out) - ref) - own * (np.abs(ref) + bound)
    return (got / bound).max(), (np.abs(U.host(lse) - ref_lse) / (e + 2.0 ** -22 * np.abs(ref_lse))).max()


CASES = {
    "one_token": dict(ctx=[700], n=[1], heads=(1, 1)),
    "tree": dict(ctx=[5, 0, 140], n=[9, 64, 33], heads=(4, 2), tree=True),
    "chain128": dict(ctx=[70], n=[128], heads=(2, 1)),
    "d64": dict(ctx=[33, 200, 0], n=[3, 7, 33], heads=(6, 2), D=64),
    "ragged": dict(ctx=[1, 900, 17, 64, 333, 2], n=[3, 1, 10, 2, 5, 7], heads=(8, 2)),
    "long": dict(ctx=[20000, 777], n=[2, 1], heads=(2, 1)),
    "four_waves": dict(ctx=[(37 * i) % 200 for i in range(70)], n=[1 + i % 3 for i in range(70)], heads=(8, 8)),
    "halves": dict(ctx=[(37 * i) % 200 for i in range(64)], n=[2 + i % 9 for i in range(64)], heads=(64, 8)),
}


@pytest.mark.parametrize("spread", [0, 3])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_as_accurate_as_stated(name, f32, spread):
    c = U.batch(121, **CASES[name])
    results, lse = ratio(c, U.quant_pools(c, spread), f32)
    print(f"{name} f32={f32} spread={spread}: results {results:.3f}, lse {lse:.3f} of the bound")
    assert results <= 1.0 and lse <= 1.0


def test_weights_that_are_subnormal_together_with_a_large_one():
    """A position far ahead of 8000 others, whose weights are 2^-22 to 2^-34 of its own, and whose values are alike."""
    c = U.batch(122, ctx=[8000], n=[1], heads=(1, 1), rotary=0)
    pools = list(U.quant_pools(c, spread=0))
    c["q"][0, 0] = 0.0
    c["q"][0, 0, :16] = 1.0
    pools[0][:] = 0
    pools[0][c["table"][0, 3], 0, 0, 5] = R.encode_e4m3(448.0)                    # score 16 * 448 * scale / sqrt(128)
    for gap in (16, 20, 23):                                                      # ... in nats: 23, 29, 33 bits
        pools[2][:] = np.float32(2.0 ** -5)
        c["q"][0, 0, :16] = U.bf16(gap * np.sqrt(128.0) / (16 * 448.0 * 2.0 ** -5))
        pools[1][:] = R.encode_e4m3(100.0)
        results, lse = ratio(c, pools, True)
        print(f"gap {gap}: {results:.3f}, {lse:.3f}")
        assert results <= 1.0 and lse <= 1.0
