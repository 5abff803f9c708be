"""Attention over the 8-bit cache for many requests and many query rows: workgroups of four waves, rows dealt to two halves of them,
groups of rows, contexts cut between workgroups, and what can go wrong where they meet."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import cache_util as U
from paper_2503_10325_amd import binding as sv
from test_gpu_attn_quant import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sv.lib()


def ragged(seed, B, top, least, most, long=()):
    rng = np.random.default_rng(seed)
    ctx = rng.integers(0, top + 1, B)
    ctx[:len(long)] = long
    return dict(ctx=ctx, n=rng.integers(least, most + 1, B))


def plan(c, f32=False):
    return sv.spec_describe_attn_quant_plan(sv.make_attn_desc(len(c["ctx"]), *c["heads"], c["D"], c["total"], int(c["n"].max()),
                                                              c["table"].shape[1], 0, 0.0, sv.SPEC_F32 if f32 else sv.SPEC_BF16))


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_four_waves(D, f32):
    """More than 512 (request, KV head) pairs, one context so long that it is cut."""
    c = U.batch(31, heads=(8, 8), D=D, **ragged(31, 70, 150, 0, 3, long=(4000, 0, 700)))
    assert ", 4>" in plan(c, f32)
    check(c, U.quant_pools(c), f32)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("f32", [False, True])
def test_rows_in_two_halves(f32, tree):
    """16 to 80 rows (fp32: more than 48) of one call: some requests fit a wave, the others go to two halves; two contexts are cut."""
    c = U.batch(32, heads=(64, 8), tree=tree, **ragged(32, 64, 90, 2, 10, long=(1500, 1200, 33)))
    assert ": 96 query rows" in plan(c, f32)
    check(c, U.quant_pools(c), f32)


def test_rows_in_two_halves_d64():
    c = U.batch(33, heads=(48, 16), D=64, tree=True, **ragged(33, 32, 60, 20, 40, long=(800,)))
    check(c, U.quant_pools(c), False)


def test_groups_of_two_halves():
    """1024 rows per KV head: eight groups of 128."""
    c = U.batch(34, heads=(64, 8), tree=True, ctx=[300, 0, 17, 40, 99, 128, 5, 64], n=[128, 128, 1, 100, 128, 17, 128, 64])
    assert ": 128 query rows at a time, 8 group(s)" in plan(c)
    check(c, U.quant_pools(c), False)


@pytest.mark.parametrize("f32", [False, True])
def test_nan_among_drafts_of_two_halves(f32):
    """A request of 80 rows, whose context is cut, holds a draft with a NaN value, and slots of NaN behind its last draft: the rows that see
    the draft are NaN in that dimension, nothing else is."""
    spec = ragged(35, 64, 30, 10, 10, long=(1400,))
    c = U.batch(35, heads=(64, 8), tree=True, **spec)
    c["parent"][:10] = [-1, 0, 0, 1, 1, 2, 3, -1, 7, 8]
    pools = list(U.quant_pools(c))
    at = lambda pos: (c["table"][0, pos // 16], pos % 16)
    page, slot = at(1400 + 1)
    pools[1][page, 3, 77, slot] = 0x7f
    page, slot = at(1400 + 9)
    pools[0][page, :, :, slot + 1:], pools[1][page, :, :, slot + 1:] = 0x7f, 0xff
    got = check(c, pools, f32)
    rows = [1, 3, 4, 6]                                                   # node 1 and its descendants
    assert np.isnan(got[rows, 24:32, 77]).all() and np.isnan(got).sum() == len(rows) * 8


def test_same_bits_whoever_is_last():
    c = U.batch(36, heads=(16, 4), **ragged(36, 20, 2500, 1, 6))
    pools = U.quant_pools(c)
    d = U.Device(c, quant=pools)
    first = [x.clone() for x in d.attend(d.q, True)]
    for _ in range(20):
        d.out.fill_(7.0)
        again = d.attend(d.q, True)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_long_and_short_contexts_on_one_head():
    c = U.batch(37, ctx=[30000, 5, 0, 12000, 31], n=[2, 1, 3, 4, 0], heads=(4, 1))
    check(c, U.quant_pools(c), True)


def test_a_thousand_requests():
    """More requests than one batch of 64 in every workgroup, alike and not."""
    c = U.batch(38, heads=(1, 1), D=64, ctx=[40] * 300 + [(11 * i) % 70 for i in range(700)], n=[1] * 300 + [i % 2 for i in range(700)])
    check(c, U.quant_pools(c), False)


def test_contexts_far_behind_the_table():
    """A context length that the block table has no room for: what it has room for is seen."""
    c = U.batch(39, ctx=[60, 60], n=[3, 2], heads=(2, 1), rotary=0)
    c["ctx"] = np.array([500000, 60], dtype=np.int32)
    check(c, U.quant_pools(c), True)


@pytest.mark.parametrize("B", [1, 3, 5, 7, 8, 9, 31, 33, 40, 63, 65])
def test_alike_requests(B):
    """As many pieces for each of alike requests, for numbers that divide nothing."""
    c = U.batch(40 + B, ctx=[450] * B, n=[2] * B, heads=(2, 1))
    check(c, U.quant_pools(c), False)


@pytest.mark.parametrize("heads", [100, 130, 300])
def test_as_many_heads_as_workgroups(heads):
    """Few ranges per KV head, or one: whole requests and no workspace then."""
    c = U.batch(50, heads=(heads, heads), D=64, ctx=[70, 0, 300], n=[2, 1, 3])
    assert (sv.spec_verify_attn_quant_workspace_size(sv.make_attn_desc(3, heads, heads, 64, 6, 3, c["table"].shape[1])) == 0) == (heads > 128)
    check(c, U.quant_pools(c), False)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("heads,n", [((1024, 1), [3]), ((100, 1), [128, 1]), ((75, 3), [40])])
def test_many_query_heads_per_kv_head(heads, n, f32):
    c = U.batch(51, heads=heads, D=64, ctx=[70, 5][:len(n)], n=n, tree=True)
    check(c, U.quant_pools(c), f32)


def test_units_in_chunks():
    """A block table with room for so many tokens that the cost of the batch is counted in chunks of units."""
    c = U.batch(52, heads=(64, 1), ctx=[300, 2500], n=[128, 100], tree=True)
    wide = np.full((2, 1 << 21), -1, dtype=np.int32)
    wide[:, :c["table"].shape[1]] = c["table"]
    c["table"] = wide
    check(c, U.quant_pools(c), False)
