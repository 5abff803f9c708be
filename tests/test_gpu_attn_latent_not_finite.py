"""Infinite latents in positions that rows see: their score may be -infinity, a weight of 0, and 0 times infinity is no number all the same."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import latent_util as U
from latent_rows import Device
from oracle import latent as R

pytestmark = pytest.mark.gpu

COLUMN = 100
CTX, N = 101, 12


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_10325_amd import binding
    binding.lib()


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("bad", [np.inf, -np.inf])
@pytest.mark.parametrize("where", ["draft", "last_draft", "beside_drafts", "context", "beside_a_page_that_is_none"])
@pytest.mark.parametrize("C,rope", [(512, 64), (256, 32)])
@pytest.mark.parametrize("at_a_time", [16, 32, 64, 128])
def test_a_latent_that_is_infinite(at_a_time, C, rope, where, bad, f32):
    """What the definition makes NaN is NaN, of rows that see the latent (of a draft, perhaps more of such a row); other rows keep their bits; the
    log-sum-exp stays finite where the definition's does."""
    c = U.batch(51, ctx=[CTX], n=[N], H=12, C=C, rope=rope, tree=True)
    at = {"draft": CTX + 4, "last_draft": CTX + N - 1, "beside_drafts": 98, "context": 40, "beside_a_page_that_is_none": 20}[where]
    if where == "beside_a_page_that_is_none":
        c["table"][0, 0] = -1
    clean = c["pool"].copy()
    c["pool"][c["table"][0, at // 16], at % 16, COLUMN] = bad
    out, lse = (U.host(x) for x in Device(c, at_a_time, f32=f32).attend())
    want, want_lse = (U.host(x) for x in Device(dict(c, pool=clean), at_a_time, f32=f32).attend())
    ref, ref_lse = R.attend(c, c["ql"], c["pool"], C, c["softmax"])[:2]
    _, _, _, A, L = R.attend(c, c["ql"], clean, C, c["softmax"])
    _, sees = R.visible(c, 0, c["held"])
    hit = sees[:, at]
    zero = np.isfinite(ref_lse)[hit]                             # rows and heads that give it no weight, of those that see it
    assert hit.any() and zero.any() and not zero.all() and np.isnan(ref[hit][..., COLUMN]).all()
    assert np.all(np.isnan(out) | ~np.isnan(ref))
    assert np.array_equal(out[~hit], want[~hit]) and np.array_equal(lse[~hit], want_lse[~hit])
    e = (2.0 ** -17 * (1 + A) + 2.0 ** -26 * L + 2.0 ** -22 * np.abs(ref_lse))[hit][zero]
    assert np.all(np.abs(lse - ref_lse)[hit][zero] <= e) and np.isnan(lse[hit][~zero]).all()
