"""Attention over the cache of latents against the 64-bit reference, more accurate than its header says.

For a row that sees L positions with weights w, A the largest scale * sum_i |q_i k_i| among them:

    |out - exact| <= (t + e) sum w |c|  (+ half a step of the result's type),   |lse - exact| <= e + 2^-22 |lse|,
    t = 2^-8 for bf16 results, 0 for fp32 ones.

t is half a step of a weight in bf16 (three terms hold all of fp32).  The header's e is 2^-17 (1 + A) + 2^-26 L: a score is a sum of exact products in up
to 36 steps, rounded to fp32 after each (2^-24 of at most A), then multiplied and subtracted (2^-24 A each), in a weight and in the sum it is divided by:
76 * 2^-24 A; the exponential and the merges a few 2^-22; results in up to 3 L / 16 steps, sums of weights in L / 32, 2^-24 each: 3.5 * 2^-28 L.  Roundings are of
either sign, and of n of them about the square root of n remains: the tests hold all kernels to e = 2^-19 (1 + A) + 2^-28 L.
"""
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


class Device(U.Device):
    """With the block table widened, by columns that hold no pages, until there is more to be done for every request than `least` groups of 16 rows x 64
    tokens: the kernels of 16, 32, 64 and 128 rows."""
    least = 0

    def __init__(self, c, **more):
        groups = len(c["ctx"]) * -(-int(c["n"].max()) * c["H"] // 16)
        columns = 4 * (self.least // groups + 1) if self.least else 0
        spare = np.full((len(c["ctx"]), max(0, columns - c["table"].shape[1])), -1, dtype=np.int32)
        super().__init__(dict(c, table=np.concatenate([c["table"], spare], 1)), **more)


@pytest.fixture(params=[0, 3000, 6000, 12000], ids=lambda least: f"above{least}", autouse=True)
def least(request, monkeypatch):
    monkeypatch.setattr(Device, "least", request.param)


def ratio(c, f32=False, softmax=0.0, pool=None):
    """The largest error by its bound, of results and of log-sum-exp; rows that see nothing and rows behind are checked for what they have to be."""
    d = Device(c, f32=f32, softmax=softmax)
    out, lse = (U.host(x) for x in d.attend())
    ref, ref_lse, size, A, L = R.attend(c, c["ql"], c["pool"] if pool is None else pool, c["C"], softmax or c["softmax"])
    m = c["total"]
    assert np.all(out[m:] == 7.0) and np.all(lse[m:] == 7.0)
    none = L[:m] == 0
    assert np.all(out[:m][none] == 0) and np.all(lse[:m][none] == -np.inf)
    e = 2.0 ** -19 * (1 + A) + 2.0 ** -28 * L
    own, t = (2.0 ** -24, 0.0) if f32 else (2.0 ** -8, 2.0 ** -8)
    bound = (t + e)[..., None] * size + 1e-30
    got = (np.abs(out - ref) - own * (np.abs(ref) + bound))[:m][~none] / bound[:m][~none]
    of_lse = (np.abs(lse - ref_lse)[:m] / (e + 2.0 ** -22 * np.abs(ref_lse))[:m])[~none]
    assert not np.isnan(got).any() and not np.isnan(of_lse).any()
    return got.max(initial=0), of_lse.max(initial=0)


def check(c, **more):
    results, lse = ratio(c, **more)
    print(f"results {results:.3f}, lse {lse:.3f} of the bound")
    assert results <= 1.0 and lse <= 1.0


CASES = {
    "one_token": dict(ctx=[700], n=[1], H=1),
    "first_token": dict(ctx=[0], n=[1], H=3),
    "sixteen_rows": dict(ctx=[5, 31, 64, 100, 0], n=[1, 1, 1, 1, 1], H=16),
    "thirtytwo_rows": dict(ctx=[33, 200, 0, 65], n=[2, 1, 2, 2], H=16),
    "sixtyfour_rows": dict(ctx=[33, 200, 0, 47], n=[3, 5, 1, 4], H=13),
    "fifty_rows": dict(ctx=[33, 200, 0, 47, 700], n=[3, 5, 1, 4, 2], H=10, tree=True),
    "tree": dict(ctx=[5, 0, 140], n=[9, 64, 33], H=5, tree=True),
    "chain128": dict(ctx=[70], n=[128], H=2),
    "ragged": dict(ctx=[1, 900, 17, 64, 333, 2], n=[3, 1, 10, 2, 5, 7], H=20),
    "many": dict(ctx=[(37 * i) % 200 for i in range(150)], n=[i % 4 for i in range(150)], H=8),
    "many_of_many_rows": dict(ctx=[(53 * i) % 150 for i in range(140)], n=[(i % 7) // 2 for i in range(140)], H=50),
    "long": dict(ctx=[20000, 777], n=[2, 1], H=4),
}


@pytest.mark.parametrize("C,rope", [(512, 64), (256, 32)])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_as_accurate_as_stated(name, f32, C, rope):
    check(U.batch(21, **CASES[name], C=C, rope=rope), f32=f32)


@pytest.mark.parametrize("C,rope", [(512, 32), (256, 64)])
@pytest.mark.parametrize("H,n", [(7, 1), (7, 4), (30, 2), (50, 7)])
def test_the_other_widths(C, rope, H, n):
    check(U.batch(22, ctx=[100, 17, 0], n=[n, 1, n], H=H, C=C, rope=rope, rows_behind=3))
    check(U.batch(23, ctx=[100, 17, 0], n=[n, 1, n], H=H, C=C, rope=rope, tree=True), f32=True)


@pytest.mark.parametrize("past", [-17, -16, -15, -1, 0, 1, 15, 16, 17])
@pytest.mark.parametrize("n,H", [(1, 128), (30, 4), (3, 5), (1, 16)])
def test_ends_around_tiles(past, n, H):
    """The drafts start, and end, at every place around a tile's border."""
    check(U.batch(24, ctx=[64 + past, 128 + past - n], n=[n, n], H=H, tree=n > 3))


@pytest.mark.parametrize("H", [16, 48])
def test_scores_that_grow_and_shrink(H):
    """References that move by more than fp32's range of exponents, upwards again and again."""
    for f32 in (False, True):
        for sign in (1.0, -1.0):
            c = U.batch(25, ctx=[600], n=[3], H=H, spread=0.0)
            for pg in range(c["held"]):
                place = np.where(c["table"][0] == pg)[0]
                if len(place):
                    c["pool"][pg] = U.bf16(c["pool"][pg] * 0.05 + sign * 0.02 * place[0] * np.sign(c["ql"][0, 0]))
            check(c, f32=f32)
            check(c, f32=f32, softmax=1.0)


def test_other_scales():
    c = U.batch(26, ctx=[100, 31], n=[2, 5], H=6)
    check(c, softmax=0.01)
    check(c, softmax=1.0, f32=True)


@pytest.mark.parametrize("H", [16, 48])
def test_pages_that_are_none(H):
    c = U.batch(27, ctx=[200, 40, 5, 64], n=[3, 2, 2, 1], H=H)
    c["table"][0, 1] = -1
    c["table"][0, 12] = c["held"]
    c["table"][1, :] = -1                                        # rows that see nothing at all
    c["table"][2, 0] = 2 ** 31 - 1
    for f32 in (False, True):
        check(c, f32=f32)
    c = U.batch(28, ctx=[200, 40], n=[3, 2], H=40)
    c["table"] = c["table"][:, :5].copy()                        # pages behind the table
    check(c)
    c = U.batch(29, ctx=[0], n=[4], H=4, tree=True)              # the drafts' own page is none
    c["table"][0, 0] = -1
    check(c)


@pytest.mark.parametrize("H", [16, 48])
def test_slots_behind_and_pages_that_are_not_the_requests(H):
    c = U.batch(30, ctx=[37, 5, 64], n=[3, 2, 1], H=H, tree=True)
    clean = c["pool"].copy()
    used = np.zeros((c["held"], 16), dtype=bool)
    for b in range(3):
        at = np.arange(c["ctx"][b] + c["n"][b])
        used[c["table"][b, at // 16], at % 16] = True
    for bad in (np.nan, np.inf, -np.inf, 3e38):
        c["pool"] = np.where(used[..., None], clean, np.float32(bad))
        for f32 in (False, True):
            check(c, f32=f32, pool=clean)


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("H", [2, 16, 40])
def test_a_draft_that_is_not_finite(bad, H):
    """Reaches the rows that see it, and no others."""
    c = U.batch(31, ctx=[37], n=[12], H=H, tree=True)
    c["ql"] = np.abs(c["ql"])                                    # (an infinite entry then gives an infinite score)
    clean = c["pool"].copy()
    node = 4
    at = 37 + node
    c["pool"][c["table"][0, at // 16], at % 16, 100] = bad
    _, sees = R.visible(c, 0, c["held"])
    hit = sees[:, at]
    assert hit[node] and not hit[:node].any()
    d = Device(c)
    out, lse = (U.host(x) for x in d.attend())
    assert np.all(np.isnan(out[hit])) and not np.isnan(out[~hit]).any() and not np.isnan(lse[~hit]).any()
    e = Device(dict(c, pool=clean))
    want, want_lse = (U.host(x) for x in e.attend())
    assert np.array_equal(out[~hit], want[~hit]) and np.array_equal(lse[~hit], want_lse[~hit])


def test_a_query_that_is_not_finite_stays_alone():
    c = U.batch(32, ctx=[100], n=[3], H=50)
    c["ql"][1, 7, 3], c["ql"][2, 0, 570] = np.nan, np.inf
    out = U.host(Device(c).attend()[0])
    bad = np.isnan(out).any(-1)
    assert bad[1, 7] and bad[2, 0] and bad.sum() == 2


def test_a_context_entry_that_is_not_finite():
    c = U.batch(33, ctx=[100], n=[2], H=3)
    c["pool"][c["table"][0, 1], 3, 7] = np.nan
    assert np.all(np.isnan(U.host(Device(c).attend()[0])))


def test_without_lse_and_twice_the_same():
    c = U.batch(34, ctx=[3000, 64, 900], n=[3, 1, 2], H=16)
    d = Device(c)
    a = d.attend()[0].clone()
    d.lse.fill_(7.0)
    d.workspace.fill_(0x3c)
    b = d.attend(lse=False)[0]
    assert torch.equal(a, b) and torch.all(d.lse == 7.0)
