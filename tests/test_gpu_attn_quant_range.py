"""Attention over the 8-bit cache at the ends of what it takes: scales of V as far apart as they can be, which may not reach the weights' sum,
and so large that results are near the end of fp32's range."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import cache_util as U
from test_gpu_attn_quant import check

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
