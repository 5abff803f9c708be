"""The two per-head products of the absorbed form against the 64-bit reference."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import latent_util as U
from oracle import latent as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_10325_amd import binding
    binding.lib()


def check_absorb(c, **more):
    got = U.host(U.Device(c, **more).absorb())
    true = R.absorb(c, c["q"], c["w_key"])
    size = np.einsum("thn,hnc->thc", np.abs(c["q"][..., :c["nope"]]).astype(np.float64), np.abs(c["w_key"]).astype(np.float64))
    C, m = c["C"], c["total"]
    assert U.product_close(got[:m, :, :C], true[:m, :, :C], size[:m], c["nope"])
    assert U.rotated_close(got[:m, :, C:], true[:m, :, C:], c["scale"] * c["q"][:m, :, c["nope"]:])
    assert np.all(got[m:] == 7.0)


def check_expand(c, **more):
    got = U.host(U.Device(c, **more).expand())
    true, m = R.expand(c["x"], c["w_value"]), c["total"]
    size = R.expand(np.abs(c["x"]), np.abs(c["w_value"]))
    assert U.product_close(got[:m], true[:m], size[:m], c["C"])
    assert np.all(got[m:] == 7.0)


CASES = {
    "one": dict(ctx=[9], n=[1], H=1),
    "sixteen": dict(ctx=[9, 100], n=[7, 9], H=3),
    "seventeen": dict(ctx=[9, 100], n=[8, 9], H=16),
    "drafts": dict(ctx=[5, 0, 1000, 17], n=[64, 1, 30, 0], H=5),
    "many": dict(ctx=[(7 * i) % 40 for i in range(150)], n=[(3 * i) % 7 for i in range(150)], H=2),
    "pieces": dict(ctx=[3] * 9, n=[120] * 9, H=1),
}


@pytest.mark.parametrize("C,rope,nope,value", [(512, 64, 128, 128), (512, 32, 64, 64), (256, 64, 128, 64), (256, 32, 64, 128)])
@pytest.mark.parametrize("name", list(CASES))
def test_sizes(name, C, rope, nope, value):
    c = U.batch(11, **CASES[name], C=C, rope=rope, nope=nope, value=value, interleaved=name != "drafts")
    check_absorb(c)
    check_expand(c)


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("behind", [1, 40])
def test_rows_behind_and_strides(apart, behind):
    c = U.batch(12, ctx=[40, 3], n=[10, 5], H=9, rows_behind=behind)
    check_absorb(c, apart=apart)
    check_expand(c, apart=apart)


def test_rows_behind_that_are_not_finite():
    c = U.batch(13, ctx=[40], n=[9], rows_behind=9)
    c["q"][9:], c["x"][9:] = np.nan, np.inf
    check_absorb(c)
    check_expand(c)


def test_a_row_that_is_not_finite_stays_alone():
    c = U.batch(14, ctx=[40], n=[20])
    c["q"][3, 1, 5], c["x"][4, 2, 500] = np.nan, np.nan
    d = U.Device(c)
    a, e = U.host(d.absorb()), U.host(d.expand())
    assert np.all(np.isnan(a[3, 1, :512])) and np.isnan(a).sum() == 512
    assert np.all(np.isnan(e[4, 2])) and np.isnan(e).sum() == 128


def test_trees_and_positions():
    check_absorb(U.batch(15, ctx=[40, 3], n=[64, 128], H=11, tree=True, scale=0.75, interleaved=True))
    pos = np.array([0, 1000000, 5, 5, 131071, 2, -3], dtype=np.int32)
    check_absorb(U.batch(16, ctx=[10, 20], n=[4, 3], positions=pos, theta=500000.0))


def test_no_rows_at_all():
    c = U.batch(17, ctx=[10, 20], n=[0, 0], rows_behind=3)
    d = U.Device(c)
    assert torch.all(d.absorb() == 7) and torch.all(d.expand() == 7) and torch.all(d.attend()[0] == 7)
    before = d.pool.clone()
    assert torch.equal(d.append(), before)
