"""Compaction of the 8-bit cache where lengths and offsets are not those of a cache in order: near 2^31, below 0; prompts and
other linear requests of more than 128 tokens."""
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


def compacted(c, pools, stop):
    """Pools and scales after the call, and the lengths; -5 where none is written."""
    d = U.Device(c, quant=pools)
    new_len = d.compact(torch.from_numpy(np.asarray(stop, dtype=np.int32)).cuda())
    torch.cuda.synchronize()
    return [U.host(x) for x in (d.k_pool, d.v_pool, d.k_scale, d.v_scale)], U.host(new_len)


def test_lengths_near_the_end_of_32_bits():
    """No page holds those places: nothing moves, and the length stays below 2^31."""
    c = U.batch(101, ctx=[20, 20, 20], n=[100, 9, 40], heads=(2, 2), tree=True)
    for o, m in ((0, 100), (100, 9), (109, 40)):
        c["parent"][o:o + m] = [max(i - 2, -1) for i in range(m)]
    pools = U.quant_pools(c)
    c["ctx"] = np.array([2**31 - 1, 2**31 - 16, 2**31 - 30], dtype=np.int32)
    after, new_len = compacted(c, pools, [99, 8, 39])
    assert all(np.array_equal(x, y) for x, y in zip(after, pools))
    assert new_len.tolist() == [2**31 - 1, 2**31 - 16 + 5, 2**31 - 30 + 20]


def test_negative_offsets_are_no_tokens():
    """As for attention and appending; the request behind it is compacted as ever."""
    c = U.batch(102, ctx=[20, 35], n=[9, 11], heads=(2, 2), tree=True)
    c["parent"][9:] = [max(i - 2, -1) for i in range(11)]
    pools = U.quant_pools(c)
    *want, want_len = R.compact_quant(c, *pools, [-1, 10])
    c["offsets"][0] = -2**31
    after, new_len = compacted(c, pools, [8, 10])
    assert all(np.array_equal(x, y) for x, y in zip(after, want))
    assert np.array_equal(new_len, want_len)


def test_long_linear_requests():
    """Nothing moves, the length grows to the last accepted token."""
    c = U.batch(103, ctx=[5, 0, 7, 9, 40], n=[300, 1000, 129, 128, 200], heads=(2, 1))
    pools = U.quant_pools(c)
    stop = [250, 999, 128, 127, 200]                                      # (no token 200 of the last)
    *want, want_len = R.compact_quant(c, *pools, stop)
    after, new_len = compacted(c, pools, stop)
    assert all(np.array_equal(x, y) for x, y in zip(after, want)) and all(np.array_equal(x, y) for x, y in zip(want, pools))
    assert np.array_equal(new_len, want_len) and new_len.tolist() == [256, 1000, 136, 137, 40]


@pytest.mark.parametrize("tree", [False, True])
def test_negative_lengths_stay(tree):
    c = U.batch(104, ctx=[20, 35], n=[9, 11], heads=(2, 2), tree=tree)
    pools = U.quant_pools(c)
    *want, want_len = R.compact_quant(c, *pools, [-1, 10])
    c["ctx"][0] = want_len[0] = -3
    after, new_len = compacted(c, pools, [8, 10])
    assert all(np.array_equal(x, y) for x, y in zip(after, want))
    assert np.array_equal(new_len, want_len)
