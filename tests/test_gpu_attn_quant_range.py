"""Attention over the 8-bit cache at the ends of what it takes: scales of V as far apart as they can be, which may not reach the weights' sum,
and so large that results are near the end of fp32's range; scores next to none, and so large that one position is all that counts."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import cache_util as U
from oracle import cache as R
from test_gpu_attn_quant import check, values_bound

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_10325_amd import binding
    binding.lib()


SPECS = {
    "one_request": dict(ctx=[120], n=[2], heads=(1, 1)),
    "d64": dict(ctx=[200, 31], n=[3, 1], heads=(4, 2), D=64),
    "units_in_turn": dict(ctx=[300 + i for i in range(70)], n=[1] * 70, heads=(8, 8), D=64),
}


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("spec", list(SPECS))
@pytest.mark.parametrize("least,gap", [(-100, 36), (-100, 121), (-100, 140), (-60, 150), (-100, 160), (-100, 200)])
def test_pages_of_zeros_beside_large_values(least, gap, spec, f32):
    """A page of zeros has the least scale; its weights count in the sum whatever the scale of the others."""
    c = U.batch(91, **SPECS[spec])
    pools = list(U.quant_pools(c, spread=0))
    large = c["rng"].random(pools[3].shape) < 0.3
    large[c["table"][0, 1]] = True
    pools[3][...] = np.where(large, np.float32(2.0) ** np.float32(least + gap), np.float32(2.0) ** np.float32(least))
    pools[1][~large] = 0
    check(c, pools, f32)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("spec", list(SPECS))
def test_scales_of_any_size(spec, f32):
    c = U.batch(92, **SPECS[spec])
    pools = list(U.quant_pools(c, spread=0))
    pools[3][...] = np.exp2(c["rng"].integers(-100, 101, pools[3].shape)).astype(np.float32)
    check(c, pools, f32)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("spec", list(SPECS) + ["cut"])
def test_largest_values(spec, f32):
    """Entries up to 448 2^119, 0.87 of the largest fp32 number: sums over the tokens would be beyond it, their mean is not."""
    c = U.batch(93, **(SPECS[spec] if spec in SPECS else dict(ctx=[3000], n=[3], heads=(2, 1))))
    pools = list(U.quant_pools(c, spread=0))
    pools[3][c["rng"].random(pools[3].shape) < 0.7] = np.float32(2.0 ** 119)
    assert np.isfinite(check(c, pools, f32)).all()


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("scale", [1e-16, 1e-30, 1e-44])
def test_next_to_no_scale(scale, f32):
    """Every score is next to 0, of pages of zeros too, whose scale times the softmax's is below fp32: the values' mean, of the positions that a row
    sees."""
    c = U.batch(94, ctx=[37, 90, 0], n=[6, 5, 9], heads=(4, 2), tree=True, rotary=0)
    pools = list(U.quant_pools(c))
    zeros = c["rng"].random(pools[2].shape) < 0.6
    zeros[c["table"][0, 2]] = True                                        # (a page of drafts)
    pools[0][zeros], pools[2][zeros] = 0, np.float32(2.0 ** -100)
    d = U.Device(c, quant=pools)
    out, lse = d.attend(d.q, f32, scale=scale)
    ref, ref_lse = R.attend(c, c["q"], *pools, scale=scale)
    assert U.attn_close(U.host(out), ref, values_bound(c, pools), f32)
    assert np.all(np.abs(U.host(lse) - ref_lse) <= 2.0 ** -19 * np.maximum(np.abs(ref_lse), 8.0))


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("spec", list(SPECS))
def test_scores_of_millions(spec, f32):
    """Up to 2^23, positions apart by more than their rounding (2^-24 of the largest, a few times): a row's result is the value of the one
    that is ahead, its log-sum-exp that score."""
    c = U.batch(95, **SPECS[spec], rotary=0)
    pools = U.quant_pools(c, spread=0)
    c["q"] = U.bf16(c["q"] * 2.0 ** 20)
    d = U.Device(c, quant=pools)
    out, lse = d.attend(d.q, f32)
    ref, ref_lse = R.attend(c, c["q"], *pools)
    assert 2.0 ** 20 < np.abs(ref_lse).max() < 2.0 ** 23
    assert np.abs(ref_lse - top_score(c, pools)).max() < 1e-6
    assert np.all(np.abs(U.host(lse) - ref_lse) <= 2.0 ** -18 * np.abs(ref_lse).max())
    assert U.attn_close(U.host(out), ref, values_bound(c, pools), f32)


def top_score(c, pools):
    """The largest score of every row, in 64 bits."""
    top = np.zeros((c["total"], c["heads"][0]))
    G = c["heads"][0] // c["heads"][1]
    for b in range(len(c["ctx"])):
        for i in range(c["n"][b]):
            at = np.arange(c["ctx"][b] + i + 1)
            page = c["table"][b, at // 16]
            k = R.E4M3[pools[0][page, :, :, at % 16]].reshape(len(at), -1, c["D"]) * pools[2][page][..., None]
            for h in range(c["heads"][0]):
                top[c["offsets"][b] + i, h] = (k[:, h // G] @ c["q"][c["offsets"][b] + i, h].astype(np.float64)).max() / np.sqrt(c["D"])
    return top
