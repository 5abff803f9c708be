"""What the cache operators refuse, on the host, before anything is launched; and the binding's own checks."""
import ctypes
import os

import numpy as np
import pytest

from oracle import cache as R
from paper_2503_10325_amd import binding as sv

pytestmark = pytest.mark.skipif(not os.path.exists(sv.LIB_PATH), reason="libspecverify.so not built")
NULL, SHAPE, UNSUPPORTED, WORKSPACE = -1, -2, -3, -4
OK = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, total_q=8, max_q_per_req=4, max_pages_per_req=10, num_pages=30, rotary_dim=64)
P = 1 << 20                                  # stands for an aligned device pointer: a refused call does not follow it


@pytest.mark.parametrize("quant", [False, True])
def test_append(quant):
    def call(q=P, qs=1024, k=P, ks=256, v=P, vs=256, inv=P, pos=None, kp=P, vp=P, scale=P, bt=P, ctx=P, off=P, parent=None, out=P, **d):
        desc = sv.make_append_desc(**{**OK, **d})
        head = (ctypes.byref(desc), q, qs, k, ks, v, vs, inv, pos, kp, vp)
        tail = (bt, ctx, off, parent, out, None)
        if quant:
            return sv.lib().spec_append_kv_quant(*head, scale, scale, *tail)
        return sv.lib().spec_append_kv(*head, *tail)

    for missing in ("k", "v", "inv", "kp", "vp", "bt", "ctx", "off"):
        assert call(**{missing: None}) == NULL, missing
    assert call(q=None) == NULL and call(out=None) == NULL           # queries without results, results without queries
    if quant:
        assert call(scale=None) == NULL
    for bad in (dict(batch=-1), dict(num_q_heads=0), dict(num_kv_heads=0), dict(num_kv_heads=3), dict(total_q=-1), dict(num_pages=0),
                dict(max_pages_per_req=0), dict(max_q_per_req=0), dict(rotary_dim=-16), dict(rotary_dim=144),
                dict(rotary_scale=-1.0), dict(rotary_scale=float("nan")), dict(qs=1023), dict(qs=1016), dict(ks=250), dict(vs=248),
                dict(ks=260), dict(q=P + 8), dict(k=P + 2), dict(v=P + 8), dict(out=P + 8), dict(kp=P + 8), dict(vp=P + 4),
                dict(qs=1536)):
        if bad == dict(qs=1536):
            assert call(q=P, out=P, **bad) == SHAPE                      # in place, but the tokens lie apart
        else:
            assert call(**bad) == SHAPE, bad
    for bad in (dict(head_dim=96), dict(page_size=32), dict(rotary_dim=24), dict(interleaved=2), dict(num_q_heads=8192, num_kv_heads=8192, qs=1 << 20, ks=1 << 20, vs=1 << 20),
                dict(parent=P, max_q_per_req=129), dict(total_q=2**31 - 1)):
        assert call(**bad) == UNSUPPORTED, bad
    assert call(batch=0) == 0 and call(total_q=0) == 0
    lib_call = sv.lib().spec_append_kv
    assert lib_call(None, P, 1024, P, 256, P, 256, P, None, P, P, P, P, P, None, P, None) == NULL


def test_attention():
    ok = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, total_q=8, max_q_per_req=4, max_pages_per_req=10)
    need = sv.spec_verify_attn_quant_workspace_size(sv.make_attn_desc(**ok))
    assert need > 0

    def call(num_pages=30, q=P, kp=P, vp=P, ks=P, vs=P, bt=P, ctx=P, off=P, out=P, ws=P, bytes_=need, **d):
        desc = sv.make_attn_desc(**{**ok, **d})
        return sv.lib().spec_verify_attn_quant(ctypes.byref(desc), num_pages, q, kp, vp, ks, vs, bt, ctx, off, None, out, None, ws, bytes_, None)

    for missing in ("q", "kp", "vp", "ks", "vs", "bt", "ctx", "off", "out"):
        assert call(**{missing: None}) == NULL, missing
    for bad in (dict(num_pages=-1), dict(num_pages=0), dict(batch=-1), dict(num_kv_heads=3), dict(scale=-1.0), dict(q=P + 8), dict(kp=P + 8),
                dict(vp=P + 1), dict(out=P + 4), dict(ws=P + 8), dict(max_pages_per_req=0), dict(max_q_per_req=0)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(head_dim=96), dict(page_size=32), dict(max_q_per_req=129), dict(out_dtype=2), dict(num_q_heads=2 * 8192)):
        assert call(**bad) == UNSUPPORTED, bad
    assert call(ws=None) == WORKSPACE and call(bytes_=need - 1) == WORKSPACE
    assert call(batch=0) == 0 and call(total_q=0) == 0
    assert sv.spec_verify_attn_quant_workspace_size(sv.make_attn_desc(**{**ok, "head_dim": 96})) == 0
    assert "attn_quant_kernel<128, 1, 8>: 16 query rows" in sv.spec_describe_attn_quant_plan(sv.make_attn_desc(**ok))
    with pytest.raises(sv.SpecError):
        sv.spec_describe_attn_quant_plan(sv.make_attn_desc(**{**ok, "head_dim": 96}))


def test_compaction():
    def call(B=2, heads=2, D=128, page=16, width=4, pages=9, **more):
        a = dict(kp=P, vp=P, ks=P, vs=P, bt=P, ctx=P, off=P, parent=P, stop=P, new=None)
        a.update(more)
        return sv.lib().spec_compact_kv_quant(B, heads, D, page, width, pages, *a.values(), None)

    for missing in ("kp", "vp", "ks", "vs", "bt", "ctx", "off", "stop"):
        assert call(**{missing: None}) == NULL, missing
    for bad in (dict(B=-1), dict(heads=0), dict(width=-1), dict(pages=-1), dict(kp=P + 8), dict(vp=P + 4)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(D=96), dict(page=32), dict(B=65536), dict(heads=65536)):
        assert call(**bad) == UNSUPPORTED, bad
    assert call(B=0) == 0


def test_binding_refuses_other_types_and_shapes():
    torch = pytest.importorskip("torch")
    t = lambda shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    desc = sv.make_append_desc(**{**OK, "rotary_dim": 0})

    def append(q=t((8, 8, 128)), k=t((8, 2, 128)), v=t((8, 2, 128)), kp=t((30, 2, 16, 128)), bt=i32(2, 10), ctx=i32(2)):
        sv.spec_append_kv(desc, q, k, v, None, kp, kp, bt, ctx, i32(3), None, t((8, 8, 128)), stream=_Stream())

    for bad in (dict(q=t((8, 8, 128), torch.float16)), dict(kp=t((30, 2, 16, 128), torch.float32)), dict(bt=torch.zeros((2, 10), dtype=torch.int64)),
                dict(ctx=torch.zeros(2))):
        with pytest.raises(TypeError):
            append(**bad)
    for bad in (dict(q=t((8, 4, 128))), dict(k=t((9, 2, 128))), dict(v=t((8, 2, 256))[..., ::2])):
        with pytest.raises(ValueError):
            append(**bad)
    pools = [t((30, 2, 8, 16, 16), torch.uint8), t((30, 2, 128, 16), torch.uint8), t((30, 2), torch.float32), t((30, 2), torch.float32)]
    for i, bad in ((0, t((30, 2, 8, 16, 16))), (0, t((30, 2, 4, 16, 16), torch.uint8)), (2, t((30, 2))), (3, t((30, 3), torch.float32))):
        mixed = list(pools)
        mixed[i] = bad
        with pytest.raises((TypeError, ValueError)):
            sv.spec_compact_kv_quant(*mixed, i32(2, 10), i32(2), i32(3), None, i32(2), stream=_Stream())


class _Stream:
    cuda_stream = 0


# ---- the reference itself ----
def test_reference_codes_match_torch():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(4000) * 10.0 ** rng.uniform(-4, 2.4, 4000), R.E4M3[~np.isnan(R.E4M3)],
                        (R.E4M3[:126] + R.E4M3[1:127]) / 2, [0.0, -0.0, 448.0, -448.0]])
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(R.encode_e4m3(x), want)
    back = torch.from_numpy(np.arange(256, dtype=np.uint8)).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(R.E4M3, back, equal_nan=True)


def test_reference_scales():
    assert R.page_scale(448.0) == 1.0 and R.page_scale(np.nextafter(448.0, 999)) == 2.0 and R.page_scale(0.0) == 2.0 ** -100
    assert R.page_scale(224.0) == 0.5 and R.page_scale(1.0) == 2.0 ** -8


def test_millions_of_groups_of_rows():
    """More requests times groups of query rows than the cut of the batch can count in 31 bits."""
    big = dict(batch=65535, num_q_heads=1024, num_kv_heads=1, head_dim=64, total_q=65535 * 128, max_q_per_req=128, max_pages_per_req=10)
    desc = sv.make_attn_desc(**big)
    assert sv.spec_verify_attn_quant_workspace_size(desc) == 0
    rc = sv.lib().spec_verify_attn_quant(ctypes.byref(desc), 30, P, P, P, P, P, P, P, P, None, P, None, P, 1 << 40, None)
    assert rc == UNSUPPORTED
    with pytest.raises(sv.SpecError):
        sv.spec_describe_attn_quant_plan(desc)
    # a wide block table alone is no reason
    assert sv.spec_verify_attn_quant_workspace_size(sv.make_attn_desc(**{**big, "batch": 64, "max_pages_per_req": 2**31 - 1})) > 0


def test_binding_refuses_pools_that_are_not_the_descriptors():
    torch = pytest.importorskip("torch")
    t = lambda shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    desc = sv.make_append_desc(**{**OK, "rotary_dim": 0})
    rows = (t((8, 8, 128)), t((8, 2, 128)), t((8, 2, 128)), None)
    rest = (i32(2, 10), i32(2), i32(3), None, t((8, 8, 128)))
    for shape in ((29, 2, 16, 128), (30, 1, 16, 128), (30, 2, 16, 64)):
        with pytest.raises(ValueError):
            sv.spec_append_kv(desc, *rows, t(shape), t(shape), *rest, stream=_Stream())

    def quant(pages, heads, dim):
        return (t((pages, heads, dim // 16, 16, 16), torch.uint8), t((pages, heads, dim, 16), torch.uint8),
                t((pages, heads), torch.float32), t((pages, heads), torch.float32))

    attn = sv.make_attn_desc(2, 8, 2, 128, 8, 4, 10)
    for pages, heads, dim in ((29, 2, 128), (30, 1, 128), (30, 2, 64)):
        with pytest.raises(ValueError):
            sv.spec_append_kv_quant(desc, *rows, *quant(pages, heads, dim), *rest, stream=_Stream())
        if (heads, dim) != (2, 128):
            with pytest.raises(ValueError):
                sv.spec_verify_attn_quant(attn, rows[0], *quant(pages, heads, dim), *rest[:4], rest[4], stream=_Stream())
