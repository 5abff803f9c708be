"""Attention over latents of large magnitude, up to where its header says that its accuracy ends: L max |c| = 2^111."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import latent_util as U
from latent_rows import Device
from oracle import latent as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_10325_amd import binding
    binding.lib()


def batch(C, rope, rises, most):
    """Scores, in log2 units, of 0 in the first 64 tokens and of about `rises`, one after the other, in the next ones, from the shared keys alone; latents of
    magnitudes up to `most`, of either sign but more often positive, so that sums grow with the number of tokens."""
    ctx = 64 * (1 + len(rises)) + 3
    c = U.batch(41, ctx=[ctx], n=[3], H=48, C=C, rope=rope, spread=0.0)
    rng = c["rng"]
    c["ql"][:] = 0
    c["ql"][:, :, C] = 8
    per_unit = np.log(2) / (8 * c["softmax"])
    c["pool"][:] = 0
    at = np.arange(ctx + 3)
    level = np.concatenate([[0.0], rises])[np.minimum(at // 64, len(rises))]
    rows = np.zeros((ctx + 3, C + rope))
    rows[:, :C] = most * rng.uniform(0.5, 1, (ctx + 3, C)) * np.where(rng.random((ctx + 3, C)) < 0.8, 1, -1)
    rows[:, C] = level * per_unit
    cut = U.bf16(rows)
    assert np.abs(cut[:, :C]).max() * (ctx + 3) <= 2.0 ** 111
    c["pool"][c["table"][0, at // 16], at % 16] = cut
    return c


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("rises", [[0.0], [15.5], [39.0], [39.0, 78.0, 117.0]], ids=["level", "15", "39", "39-78-117"])
@pytest.mark.parametrize("C,rope", [(512, 64), (256, 32)])
@pytest.mark.parametrize("at_a_time", [16, 32, 64, 128])
def test_large_latents(at_a_time, C, rope, rises, f32):
    """Bounds as the header has them: a result is off by its rounding and (t + e) sum w |c|."""
    c = batch(C, rope, rises, 2.0 ** 111 * 0.99 / (64 * (1 + len(rises)) + 6))
    out, lse = (U.host(x) for x in Device(c, at_a_time, f32=f32).attend())
    ref, ref_lse, size, A, L = R.attend(c, c["ql"], c["pool"], C, c["softmax"])
    e = 2.0 ** -17 * (1 + A) + 2.0 ** -26 * L
    own, t = (2.0 ** -24, 0.0) if f32 else (2.0 ** -8, 2.0 ** -8)
    bound = (t + e)[..., None] * size
    assert np.isfinite(out).all()
    assert np.all(np.abs(out.astype(np.float64) - ref) <= bound + own * (np.abs(ref) + bound))
    assert np.all(np.abs(lse - ref_lse) <= e + 2.0 ** -22 * np.abs(ref_lse))
