"""GPU parity of appending keys and values to the paged cache, with rotation (spec_append_kv, spec_append_kv_quant, through
the C ABI) against the 64-bit reference."""
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


CASES = {
    "one_token": dict(ctx=[0], n=[1], heads=(1, 1)),
    "single_tokens": dict(ctx=[15, 16, 17, 0, 31, 1000], n=[1] * 6, heads=(8, 2)),
    "odd_lengths": dict(ctx=[5, 0, 33, 100], n=[7, 1, 16, 31], heads=(3, 3)),
    "some_empty": dict(ctx=[5, 0, 33, 16], n=[0, 3, 0, 0], heads=(2, 1)),
    "prompt": dict(ctx=[0, 3], n=[133, 300], heads=(4, 2)),
    "d64": dict(ctx=[5, 0, 33, 100], n=[7, 1, 16, 40], heads=(6, 2), D=64),
    "tree": dict(ctx=[5, 0, 40], n=[9, 128, 33], heads=(4, 2), tree=True),
    "tree_d64": dict(ctx=[17], n=[64], heads=(4, 4), D=64, tree=True),
    "half_rotated": dict(ctx=[9, 60], n=[20, 5], rotary=64),
    "least_rotated": dict(ctx=[9, 60], n=[20, 5], rotary=16),
    "odd_rotated": dict(ctx=[9, 60], n=[20, 5], rotary=112),
    "d64_part": dict(ctx=[9, 60], n=[20, 5], rotary=48, D=64),
    "not_rotated": dict(ctx=[9, 60], n=[20, 5], rotary=0),
    "neighbours": dict(ctx=[9, 60], n=[20, 5], interleaved=True),
    "neighbours_part": dict(ctx=[9, 60], n=[20, 5], interleaved=True, rotary=48),
    "neighbours_d64": dict(ctx=[9, 60], n=[20, 5], interleaved=True, D=64, tree=True),
    "scaled": dict(ctx=[9, 60], n=[20, 5], scale=1.25),
    "own_positions": dict(ctx=[9, 60], n=[3, 4], positions=np.array([0, 1 << 20, 5, 2**31 - 1, 7, 7, 131071], dtype=np.int32)),
    "rows_behind": dict(ctx=[9, 60], n=[20, 5], rows_behind=9),
    "rows_behind_tree": dict(ctx=[9, 60], n=[20, 5], rows_behind=40, tree=True),
    "many_requests": dict(ctx=list(range(200)), n=[(3 * i) % 5 for i in range(200)], heads=(2, 1), D=64),
    "many_heads": dict(ctx=[7], n=[18], heads=(96, 96), D=64),
}


def make(name, seed=1):
    return U.batch(seed, **CASES[name])


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_bf16_cache(name, fused):
    c = make(name)
    pools = [U.bf16(c["rng"].standard_normal((c["held"], c["heads"][1], 16, c["D"]))) for _ in range(2)]
    d = U.Device(c, fused, bf16_pools=pools)
    d.append()
    torch.cuda.synchronize()
    q, k, v = R.append(c, *pools)
    t = c["total"]
    assert U.rotated_close(U.host(d.q_out)[:t], q[:t], c["q"][:t], c["rotary"], 2.0 ** -8)
    assert np.all(U.host(d.q_out)[t:] == 7.0)
    got = U.host(d.k_pool)
    changed = np.any(k != pools[0].astype(np.float64), axis=-1)
    assert np.array_equal(got[~changed], pools[0][~changed])              # every other slot as it was
    assert U.rotated_close(got, k, np.full_like(got, np.abs(c["k"]).max()), c["rotary"], 2.0 ** -8)
    assert np.array_equal(U.host(d.v_pool), v.astype(np.float32))          # copied


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_quant_cache(name, fused):
    c = make(name, 2)
    pools = U.quant_pools(c)
    d = U.Device(c, fused, quant=pools)
    d.append()
    torch.cuda.synchronize()
    q, k, v, ks, vs, truth = R.append_quant(c, *pools)
    t = c["total"]
    assert U.rotated_close(U.host(d.q_out)[:t], q[:t], c["q"][:t], c["rotary"], 2.0 ** -8)
    assert np.all(U.host(d.q_out)[t:] == 7.0)
    assert np.array_equal(U.host(d.v_scale), vs) and np.array_equal(U.host(d.v_pool), v)
    assert np.array_equal(U.host(d.k_scale), ks)
    got = U.host(d.k_pool)
    other = got != k
    for (pg, h, slot), x in truth.items():
        # a code that differs stands for a value as near, but for the fp32 rotation of its pair
        val = R.E4M3[got[pg, h, :, slot].reshape(-1)] * ks[pg, h]
        step = R.e4m3_step(x / ks[pg, h]) * ks[pg, h]
        assert np.all(np.abs(val - x) <= step / 2 + 2.0 ** -20 * np.abs(c["k"]).max()), (pg, h, slot)
        other[pg, h, :, slot] = False
    assert not other.any()


def test_scale_grows_and_never_shrinks():
    """Committed entries are rewritten when a larger one arrives, and keep their scale when only small ones do."""
    c = U.batch(3, ctx=[5, 5], n=[2, 2], heads=(2, 2), rotary=0)
    pools = U.quant_pools(c, spread=0)
    c["k"][:2] *= 64.0
    c["v"][:2] *= 64.0
    c["k"][2:] *= 2.0 ** -10
    c["v"][2:] *= 2.0 ** -10
    d = U.Device(c, quant=pools)
    d.append()
    torch.cuda.synchronize()
    _, k, v, ks, vs, _ = R.append_quant(c, *pools)
    first, second = int(c["table"][0, 0]), int(c["table"][1, 0])
    assert np.all(ks[first] > pools[2][first]) and np.array_equal(ks[second], pools[2][second])
    for got, want in ((d.k_pool, k), (d.v_pool, v), (d.k_scale, ks), (d.v_scale, vs)):
        assert np.array_equal(U.host(got), want)
    d.append()                                                            # the same call again changes nothing
    for got, want in ((d.k_pool, k), (d.v_pool, v), (d.k_scale, ks), (d.v_scale, vs)):
        assert np.array_equal(U.host(got), want)


def test_infinities_nan_zeros_and_extremes():
    c = U.batch(4, ctx=[3, 0, 0, 0], n=[4, 2, 2, 2], heads=(1, 1), rotary=0)
    for x in (c["k"], c["v"]):
        x[0, 0, 5], x[1, 0, 7], x[2, 0, 9] = np.inf, -np.inf, np.nan
        x[4:6] = 0.0                                                      # a page of zeros
        x[6:8] *= 2.0 ** -120                                             # below the least scale
        x[8:10] = np.float32(3.3e38)                                      # beyond the largest
    pools = U.quant_pools(c)
    d = U.Device(c, quant=pools)
    d.append()
    torch.cuda.synchronize()
    _, k, v, ks, vs, _ = R.append_quant(c, *pools)
    for got, want in ((d.k_scale, ks), (d.v_scale, vs)):
        assert np.array_equal(U.host(got), want)
    for got, want in ((d.k_pool, k), (d.v_pool, v)):                      # (a NaN's sign is not specified)
        assert np.array_equal(R.E4M3[U.host(got)], R.E4M3[want], equal_nan=True)


@pytest.mark.parametrize("quant", [False, True])
def test_bad_pages_receive_nothing(quant):
    c = U.batch(5, ctx=[30, 10, 5], n=[20, 30, 4], heads=(2, 1))
    c["table"][0, 2], c["table"][1, 1] = -1, c["held"] + 5
    c["table"] = np.ascontiguousarray(c["table"][:, :3])                  # the last page of both lies behind the table
    pools = U.quant_pools(c) if quant else [U.bf16(c["rng"].standard_normal((c["held"], 1, 16, c["D"]))) for _ in range(2)]
    d = U.Device(c, **({"quant": pools} if quant else {"bf16_pools": pools}))
    d.append()
    torch.cuda.synchronize()
    if quant:
        q, k, v, ks, vs, _ = R.append_quant(c, *pools)
        assert np.array_equal(U.host(d.v_pool), v) and np.array_equal(U.host(d.k_scale), ks) and np.array_equal(U.host(d.v_scale), vs)
        untouched = ks == pools[2]
        assert np.array_equal(U.host(d.k_pool)[untouched & (vs == pools[3])], k[untouched & (vs == pools[3])])
    else:
        q, k, v = R.append(c, *pools)
        assert np.array_equal(U.host(d.v_pool), v.astype(np.float32))
    assert U.rotated_close(U.host(d.q_out), q, c["q"], c["rotary"], 2.0 ** -8)


@pytest.mark.parametrize("quant", [False, True])
def test_queries_in_place_and_without_queries(quant):
    c = U.batch(6, ctx=[30, 11], n=[20, 3], heads=(4, 2))
    pools = U.quant_pools(c) if quant else [U.bf16(c["rng"].standard_normal((c["held"], 2, 16, c["D"]))) for _ in range(2)]
    make_dev = lambda: U.Device(c, **({"quant": pools} if quant else {"bf16_pools": pools}))
    a, b, n = make_dev(), make_dev(), make_dev()
    a.append()
    b.append(q_out=b.q)
    n.append(q=None, q_out=None)
    torch.cuda.synchronize()
    assert torch.equal(a.q_out, b.q)
    for x in (b, n):
        assert torch.equal(a.k_pool, x.k_pool) and torch.equal(a.v_pool, x.v_pool)


def test_far_positions_keep_their_angles():
    """At position 2^31 - 1 an fp32 angle would be off by whole turns."""
    c = U.batch(7, ctx=[0], n=[1], heads=(1, 1), theta=1e6, positions=np.array([2**31 - 1], dtype=np.int32))
    pools = [np.zeros((c["held"], 1, 16, 128), dtype=np.float32) for _ in range(2)]
    d = U.Device(c, bf16_pools=pools)
    d.append()
    q, _, _ = R.append(c, *pools)
    assert U.rotated_close(U.host(d.q_out), q, c["q"], 128, 2.0 ** -8)
