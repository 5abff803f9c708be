"""Appending to the cache of latents against the 64-bit reference."""
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


def check(c, norm=True, **more):
    d = U.Device(c, **more)
    got = U.host(d.append(norm))
    true = R.append(c, c["latent"], c["key"], c["pool"], c["norm"] if norm else None, U.EPS)
    C = c["C"]
    written = np.any(R.append(c, c["latent"] * 0 + 1e30, c["key"] * 0 + 1e30, c["pool"]) != c["pool"], -1)
    assert np.array_equal(got[~written], c["pool"][~written])
    if norm:        # 64-bit arithmetic, rounded to fp32 and then to bf16
        assert np.all(np.abs(got[..., :C] - true[..., :C]) <= (U.HALF + 2.0 ** -23) * np.abs(true[..., :C]))
    else:
        assert np.array_equal(got[..., :C], true[..., :C])
    assert U.rotated_close(got[..., C:][written], true[..., C:][written], 2.0 * np.abs(true[..., C:][written]).max() + np.zeros_like(true[..., C:][written]))
    return got


CASES = {
    "one": dict(ctx=[0], n=[1]),
    "drafts": dict(ctx=[5, 16, 31, 100], n=[4, 1, 17, 9]),
    "prompts": dict(ctx=[0, 7, 160], n=[300, 1, 95]),
    "nothing": dict(ctx=[3, 9, 4], n=[0, 5, 0]),
    "many": dict(ctx=[(7 * i) % 40 for i in range(150)], n=[(3 * i) % 7 for i in range(150)]),
}


@pytest.mark.parametrize("C,rope", [(512, 64), (512, 32), (256, 64), (256, 32)])
@pytest.mark.parametrize("name", list(CASES))
def test_slots_and_rotation(name, C, rope):
    for norm, interleaved in ((True, True), (False, False), (True, False)):
        check(U.batch(1, **CASES[name], C=C, rope=rope, interleaved=interleaved), norm)


@pytest.mark.parametrize("apart", [False, True])
def test_trees_scaled_rotation_and_rows_behind(apart):
    check(U.batch(2, ctx=[40, 3], n=[64, 128], tree=True, scale=1.25, rows_behind=5, interleaved=True), apart=apart)


def test_given_positions():
    pos = np.array([0, 1000000, 5, 5, 131071, 2, -3], dtype=np.int32)
    check(U.batch(3, ctx=[10, 20], n=[4, 3], positions=pos, theta=500000.0))


def test_pages_that_are_none():
    c = U.batch(4, ctx=[30, 5, 16], n=[20, 40, 3], spare=2)
    c["table"][0, 2] = -1
    c["table"][1, 1] = c["held"]
    c["table"][2, 1] = 2 ** 31 - 1
    check(c)
    c = U.batch(5, ctx=[30], n=[20])
    c["table"] = c["table"][:, :2].copy()                       # a third page is behind the table
    check(c)
    c = U.batch(6, ctx=[-1, 4], n=[3, 3])                       # no request
    d = U.Device(c)
    got = U.host(d.append())
    assert np.array_equal(got[c["table"][0, 0]], c["pool"][c["table"][0, 0]]) and not np.array_equal(got, c["pool"])


def test_what_is_not_finite_and_what_is_extreme():
    c = U.batch(7, ctx=[3], n=[6])
    c["latent"][0, 5] = np.nan
    c["latent"][1, :] = 0.0
    c["latent"][2, :] = 3.0e38
    c["latent"][3, :] = 1.0e-30
    c["latent"] = U.bf16(c["latent"])
    got = U.host(U.Device(c).append())
    true = R.append(c, c["latent"], c["key"], c["pool"], c["norm"], U.EPS)
    pg = c["table"][0, 0]
    assert np.all(np.isnan(got[pg, 3, :512])) and np.all(np.isfinite(got[pg, 4:9]))
    assert np.all(np.abs(got[pg, 4:9, :512] - true[pg, 4:9, :512]) <= 1.01 * U.HALF * np.abs(true[pg, 4:9, :512]))
    assert np.all(got[pg, 4, :512] == 0)
