"""GPU parity of attention over the 8-bit cache (spec_verify_attn_quant, through the C ABI) against the 64-bit reference."""
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


def values_bound(c, pools):
    """The largest |v| of each (request, KV head), spread over the rows: [total, Hq, 1]."""
    _, v_pool, _, v_scale = pools
    out = np.zeros((c["total"], c["heads"][0], 1))
    G = c["heads"][0] // c["heads"][1]
    for b in range(len(c["ctx"])):
        pages = [p for p in c["table"][b] if 0 <= p < c["held"]]
        if pages:
            top = np.nanmax(np.abs(R.E4M3[v_pool[pages]]) * v_scale[pages][..., None, None], axis=(0, 2, 3))
            out[c["offsets"][b]:c["offsets"][b + 1], :, 0] = np.repeat(top, G)
    return out


def check(c, pools, f32, want_lse=True):
    d = U.Device(c, quant=pools)
    out, lse = d.attend(d.q, f32, want_lse)
    torch.cuda.synchronize()
    ref, ref_lse = R.attend(c, c["q"], *pools)
    t = c["total"]
    got = U.host(out)
    assert np.array_equal(np.isnan(got[:t]), np.isnan(ref[:t]))
    fine = ~np.isnan(ref[:t])
    assert U.attn_close(np.where(fine, got[:t], 0), np.where(fine, ref[:t], 0), values_bound(c, pools), f32)
    assert np.all(got[t:] == 7.0)
    if want_lse:
        gl = U.host(lse)[:t]
        same = (gl == ref_lse[:t]) | (np.isnan(gl) & np.isnan(ref_lse[:t]))
        with np.errstate(invalid="ignore"):
            near = np.abs(gl - ref_lse[:t]) <= 2.0 ** -19 * np.maximum(np.abs(ref_lse[:t]), 8.0)
        assert np.all(same | near)
    return got


CASES = {
    "one_token": dict(ctx=[0], n=[1], heads=(1, 1)),
    "single_tokens": dict(ctx=[0, 15, 16, 63, 64, 65, 700], n=[1] * 7, heads=(8, 2)),
    "chain": dict(ctx=[100, 0, 257], n=[5, 9, 64], heads=(4, 4)),
    "chain128": dict(ctx=[70], n=[128], heads=(2, 1)),
    "odd_group": dict(ctx=[33, 200], n=[3, 7], heads=(21, 3)),
    "d64": dict(ctx=[33, 200, 0], n=[3, 7, 33], heads=(6, 2), D=64),
    "tree": dict(ctx=[5, 0, 140], n=[9, 64, 33], heads=(4, 2), tree=True),
    "tree128": dict(ctx=[61], n=[128], heads=(4, 2), tree=True),
    "tree_d64": dict(ctx=[50, 3], n=[116, 2], heads=(4, 1), D=64, tree=True),
    "rows16": dict(ctx=[300], n=[16], heads=(1, 1)),
    "rows32": dict(ctx=[300], n=[8], heads=(4, 1)),
    "rows48": dict(ctx=[300], n=[6], heads=(8, 1)),
    "rows64": dict(ctx=[300], n=[8], heads=(8, 1)),
    "rows80": dict(ctx=[300, 20], n=[10, 2], heads=(16, 2)),
    "rows112": dict(ctx=[300], n=[14], heads=(8, 1)),
    "rows_1024": dict(ctx=[130], n=[128], heads=(8, 1), tree=True),
    "some_empty": dict(ctx=[33, 0, 50], n=[0, 0, 3], heads=(2, 1)),
    "ragged": dict(ctx=[1, 900, 17, 64, 333, 2], n=[3, 1, 10, 2, 5, 7], heads=(8, 2)),
    "long": dict(ctx=[4999], n=[2], heads=(2, 2)),
    "long_tree": dict(ctx=[3001], n=[21], heads=(2, 1), tree=True),
    "many_requests": dict(ctx=[(7 * i) % 90 for i in range(150)], n=[1 + i % 3 for i in range(150)], heads=(2, 1), D=64),
    "rows_behind": dict(ctx=[100, 20], n=[5, 9], heads=(4, 2), rows_behind=7),
}


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_matches_reference(name, f32):
    c = U.batch(11, **CASES[name])
    check(c, U.quant_pools(c), f32)


def test_same_bits_again_and_without_lse():
    c = U.batch(12, **CASES["ragged"])
    pools = U.quant_pools(c)
    a, b = check(c, pools, True), check(c, pools, True, want_lse=False)
    assert np.array_equal(a, b)


def test_single_tokens_with_long_split_contexts():
    c = U.batch(13, ctx=[20000, 777], n=[1, 1], heads=(4, 1))
    check(c, U.quant_pools(c), True)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("gap", [10, 20, 30])
def test_scales_far_apart(gap, f32):
    """Values of pages 2^gap apart, with the weight on the small ones: nothing is lost to the large ones."""
    c = U.batch(14, ctx=[120], n=[2], heads=(1, 1), rotary=0)
    pools = list(U.quant_pools(c, spread=0))
    big = c["table"][0, 1]
    pools[3][big] *= 2.0 ** gap
    # the large page's keys point away from the queries: a weight of exp(-60) or so
    q = c["q"][:, 0]
    q[1] = q[0]
    away = -q[0] / np.linalg.norm(q[0]) * 60.0 * np.sqrt(c["D"]) / np.linalg.norm(q[0])
    pools[2][big] = R.page_scale(np.abs(away).max())
    pools[0][big, 0] = np.repeat(R.encode_e4m3(away / pools[2][big, 0]).reshape(-1, 1, 16), 16, axis=1)
    d = U.Device(c, quant=pools)
    out, _ = d.attend(d.q, f32)
    ref, _ = R.attend(c, c["q"], *pools)
    small = np.abs(R.E4M3[pools[1]]).max() * pools[3][c["table"][0, 0]].max()
    spill = 2.0 ** gap * 448 * pools[3].min() * np.exp(-40.0)            # what the large page's own rounded weight may add
    assert np.all(np.abs(U.host(out) - ref) <= (2.0 ** -8 if not f32 else 2.0 ** -24) * np.abs(ref) + 2.0 ** (-10 if not f32 else -16) * small + spill)


def test_stale_slots_and_masked_drafts_may_hold_nan():
    """Slots behind the last draft hold NaN codes; a draft's NaN value or key reaches the rows that see it, no other."""
    c = U.batch(15, ctx=[37, 90], n=[6, 5], heads=(4, 2), tree=True)
    c["parent"][:6] = [-1, -1, 0, 1, 2, -1]
    c["parent"][6:] = [-1, 0, 0, 2, -1]
    pools = list(U.quant_pools(c))
    for b, end in ((0, 43), (1, 95)):
        pg = c["table"][b, end // 16]
        pools[0][pg, :, :, end % 16:] = 0x7f
        pools[1][pg, :, :, end % 16:] = 0xff
    at = lambda b, pos: (c["table"][b, pos // 16], pos % 16)
    pg, s = at(0, 37 + 1)                                                 # V of node 1: rows 1 and 3, dimension 5
    pools[1][pg, 0, 5, s] = 0x7f
    pg, s = at(1, 90 + 2)                                                 # K of node 2: rows 2 and 3, all of the first KV head
    pools[0][pg, 0, 3, s, 1] = 0xff
    for f32 in (False, True):
        got = check(c, pools, f32)
        nan = np.isnan(got)
        assert nan[[1, 3], 0, 5].all() and nan[[1, 3], 1, 5].all() and nan[8:10, :2].all() and not nan[:, 2:].any()
        assert nan.sum() == 4 + 2 * 2 * c["D"]


def test_nan_in_the_context_reaches_every_row():
    c = U.batch(16, ctx=[200], n=[3], heads=(2, 1))
    pools = list(U.quant_pools(c))
    pools[1][c["table"][0, 2], 0, 17, 4] = 0x7f
    got = check(c, pools, False)
    assert np.isnan(got[:, :, 17]).all() and np.isnan(got).sum() == 6


def test_bad_pages_count_as_not_there():
    c = U.batch(17, ctx=[200, 70, 3], n=[3, 4, 2], heads=(2, 1))
    c["table"][0, 3], c["table"][0, 12], c["table"][1, 0], c["table"][2, 0] = -1, c["held"], -7, 2**31 - 1
    pools = U.quant_pools(c)
    pools[1][0, :] = 0x7f                                                 # page 0, which is read in their place
    keep = [b for b in range(3) if 0 in c["table"][b]]
    if keep:
        c["table"][c["table"] == 0] = -1
    got = check(c, pools, True)
    assert np.all(got[7:9] == 0.0)                                        # the last request sees nothing


def test_table_narrower_than_the_tokens():
    c = U.batch(18, ctx=[100], n=[3], heads=(2, 1))
    c["table"] = np.ascontiguousarray(c["table"][:, :4])
    check(c, U.quant_pools(c), False)


def test_scale_argument_and_large_scores():
    """Scores of many hundreds, a single position far ahead of the others."""
    c = U.batch(19, ctx=[333], n=[4], heads=(2, 1), rotary=0)
    c["q"] *= 32.0
    pools = U.quant_pools(c)
    d = U.Device(c, quant=pools)
    out, lse = d.attend(d.q, True, scale=0.25)
    ref, ref_lse = R.attend(c, c["q"], *pools, scale=0.25)
    top = np.abs(ref_lse).max()
    assert np.all(np.abs(U.host(lse) - ref_lse) <= 2.0 ** -18 * top)
    # a weight is off by the error of its score, 2^-22 of the largest, in the exponent
    assert np.all(np.abs(U.host(out) - ref) <= (2.0 ** -16 + 2.0 ** -19 * top) * values_bound(c, pools))
