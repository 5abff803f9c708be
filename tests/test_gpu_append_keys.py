"""Keys that appending writes, slot by slot: where pages are missing, and in a decoding loop, whose attention reads the cache as it finds it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import cache_util as U
from oracle import cache as R
from test_gpu_cache_run import greedy, roomy

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_10325_amd import binding
    binding.lib()


def fresh_slots(c):
    """(page, slot) of every new token that has a page."""
    at = [(R.page_of(c["table"][b], slot // R.PAGE, c["held"]), slot % R.PAGE) for b, _, _, slot, _ in R.token_rows(c)]
    return [x for x in at if x[0] >= 0]


def check_bf16_keys(c, before, got):
    """New keys: the rotated ones, rounded once (half a step), but for fp32 rotation; every other slot as it was."""
    _, k, _ = R.append(c, before, before)
    new = np.zeros(got.shape[:1] + got.shape[2:3], dtype=bool)
    for page, slot in fresh_slots(c):
        new[page, slot] = True
    got, k, old = (x.transpose(0, 2, 1, 3) for x in (got, k, before))
    assert np.array_equal(got[~new], old[~new])
    assert U.rotated_close(got[new], k[new], np.full_like(got[new], np.abs(c["k"]).max()), c["rotary"], 2.0 ** -8)


def check_quant_keys(c, before, got):
    """New codes: within half a step of the rotated keys, but for fp32 rotation; committed ones rewritten as the scale asks; every other as it was."""
    _, k, _, ks, _, truth = R.append_quant(c, *before)
    assert len(truth) == len(set(fresh_slots(c))) * c["heads"][1] > 0
    other = got != k
    for (pg, h, slot), x in truth.items():
        val = R.E4M3[got[pg, h, :, slot].reshape(-1)] * ks[pg, h]
        step = R.e4m3_step(x / ks[pg, h]) * ks[pg, h]
        assert np.all(np.abs(val - x) <= step / 2 + (2.0 ** -20 * np.abs(c["k"]).max() if c["rotary"] else 0)), (pg, h, slot)
        other[pg, h, :, slot] = False
    assert not other.any()


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("quant", [False, True])
def test_keys_where_pages_are_missing(quant, tree):
    c = U.batch(131, ctx=[30, 10, 5], n=[20, 30, 4], heads=(4, 2), tree=tree)
    c["table"][0, 2], c["table"][1, 1] = -1, c["held"] + 5
    c["table"] = np.ascontiguousarray(c["table"][:, :3])                  # the last page of both lies behind the table
    pools = U.quant_pools(c) if quant else [U.bf16(c["rng"].standard_normal((c["held"], 2, 16, c["D"]))) for _ in range(2)]
    d = U.Device(c, **({"quant": pools} if quant else {"bf16_pools": pools}))
    d.append()
    torch.cuda.synchronize()
    assert 0 < len(fresh_slots(c)) < c["total"]
    if quant:
        check_quant_keys(c, pools, U.host(d.k_pool))
    else:
        check_bf16_keys(c, pools[0], U.host(d.k_pool))


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("heads,D", [((8, 2), 128), ((4, 4), 64)])
def test_keys_of_decoding_steps(heads, D, tree):
    """Prompts, then drafts behind what the compaction left."""
    B = 5
    c = roomy(U.batch(132, ctx=[0] * B, n=[37, 1, 16, 90, 50], heads=heads, D=D), 160)
    d = U.Device(c, quant=U.quant_pools(c))
    ctx = np.zeros(B, dtype=np.int32)
    for step in range(5):
        if step:
            new = U.batch(132 + step, ctx=ctx, n=np.random.default_rng(step).integers(1, 9, B), heads=heads, D=D, tree=tree)
            new["table"], new["held"] = c["table"], c["held"]
            pools = (d.k_pool, d.v_pool, d.k_scale, d.v_scale)
            c, d = new, U.Device(new)
            d.k_pool, d.v_pool, d.k_scale, d.v_scale = pools
        before = [U.host(x) for x in (d.k_pool, d.v_pool, d.k_scale, d.v_scale)]
        d.append()
        check_quant_keys(c, before, U.host(d.k_pool))
        if step:
            ctx = U.host(d.compact(greedy(c, d, step)[1]))
        else:
            ctx = ctx + c["n"].astype(np.int32)
    assert ctx.sum() > 194 + 5
