"""What the latent operators refuse, on the host, before anything is launched; and the binding's own checks."""
import ctypes
import os

import pytest

from paper_2503_10325_amd import binding as sv

pytestmark = pytest.mark.skipif(not os.path.exists(sv.LIB_PATH), reason="libspecverify.so not built")
NULL, SHAPE, UNSUPPORTED, WORKSPACE = -1, -2, -3, -4
OK = dict(batch=2, num_heads=8, latent_dim=512, rope_dim=64, nope_dim=128, value_dim=128, total_q=8, max_q_per_req=4, max_pages_per_req=10, num_pages=30)
P = 1 << 20                                  # stands for an aligned device pointer: a refused call does not follow it
SHAPES = [dict(batch=-1), dict(num_heads=0), dict(total_q=-1), dict(max_q_per_req=-1), dict(max_pages_per_req=-1), dict(num_pages=-1),
          dict(rotary_scale=-1.0), dict(rotary_scale=float("nan")), dict(norm_eps=-1.0), dict(norm_eps=float("nan")), dict(scale=-1.0),
          dict(scale=float("nan"))]
OTHERS = [dict(latent_dim=384), dict(rope_dim=48), dict(rope_dim=128), dict(nope_dim=96), dict(value_dim=256), dict(page_size=32), dict(interleaved=2),
          dict(out_dtype=2), dict(num_heads=1025), dict(batch=65536), dict(total_q=2**31 - 1)]


def desc(**d):
    return ctypes.byref(sv.make_latent_desc(**{**OK, **d}))


def check(call, needed, aligned, shapes, unsupported):
    for name in needed:
        assert call(**{name: None}) == NULL, name
    for name in aligned:
        assert call(**{name: P + 8}) == SHAPE, name
    for bad in SHAPES + shapes:
        assert call(**bad) == SHAPE, bad
    for bad in OTHERS + unsupported:
        assert call(**bad) == UNSUPPORTED, bad
    assert call(batch=0) == 0 and call(total_q=0) == 0


def test_append():
    def call(latent=P, ls=576, key=P, ks=576, norm=None, inv=P, pos=None, pool=P, bt=P, ctx=P, off=P, parent=None, **d):
        return sv.lib().spec_append_latent(desc(**d), latent, ls, key, ks, norm, inv, pos, pool, bt, ctx, off, parent, None)

    check(call, ["latent", "key", "inv", "pool", "bt", "ctx", "off"], ["latent", "key", "norm", "pool"],
          [dict(ls=504), dict(ls=577), dict(ks=56), dict(ks=580), dict(max_pages_per_req=0), dict(num_pages=0), dict(max_q_per_req=0)],
          [dict(parent=P, max_q_per_req=129)])
    assert sv.lib().spec_append_latent(None, P, 576, P, 576, None, P, None, P, P, P, P, None, None) == NULL


def test_absorb():
    def call(q=P, qs=8 * 192, w=P, ws=256 * 512, inv=P, pos=None, ctx=P, off=P, parent=None, out=P, **d):
        return sv.lib().spec_absorb_latent(desc(**d), q, qs, w, ws, inv, pos, ctx, off, parent, out, None)

    check(call, ["q", "w", "inv", "ctx", "off", "out"], ["q", "w", "out"],
          [dict(qs=8 * 192 - 8), dict(qs=8 * 192 + 4), dict(ws=128 * 512 - 8), dict(ws=128 * 512 + 2), dict(max_q_per_req=0)],
          [dict(parent=P, max_q_per_req=129)])
    assert sv.lib().spec_absorb_latent(None, P, 1536, P, 65536, P, None, P, P, None, P, None) == NULL


def test_attention():
    need = sv.spec_verify_attn_latent_workspace_size(sv.make_latent_desc(**OK))
    assert need > 0

    def call(q=P, pool=P, bt=P, ctx=P, off=P, parent=None, out=P, ws=P, bytes_=need, **d):
        return sv.lib().spec_verify_attn_latent(desc(**d), q, pool, bt, ctx, off, parent, out, None, ws, bytes_, None)

    check(call, ["q", "pool", "bt", "ctx", "off", "out"], ["q", "pool", "out", "ws"],
          [dict(max_pages_per_req=0), dict(num_pages=0), dict(max_q_per_req=0)], [dict(max_q_per_req=129)])
    assert call(ws=None) == WORKSPACE and call(bytes_=need - 1) == WORKSPACE
    assert sv.lib().spec_verify_attn_latent(None, P, P, P, P, P, None, P, None, P, need, None) == NULL
    for bad in SHAPES + OTHERS + [dict(max_q_per_req=129)]:
        assert sv.spec_verify_attn_latent_workspace_size(sv.make_latent_desc(**{**OK, **bad})) == 0
        with pytest.raises(sv.SpecError):
            sv.spec_describe_attn_latent_plan(sv.make_latent_desc(**{**OK, **bad}))
    for heads, pages, rows in ((4, 10, 16), (8, 10, 16), (8, 4000, 32), (8, 8000, 32), (16, 2000, 32), (16, 4000, 64), (32, 2000, 64), (32, 8000, 128)):     # 4 tokens of that many heads
        plan = sv.spec_describe_attn_latent_plan(sv.make_latent_desc(**{**OK, "num_heads": heads, "max_pages_per_req": pages}))
        assert f" {rows} query rows" in plan, plan


def test_expand():
    def call(x=P, w=P, ws=256 * 512, off=P, out=P, **d):
        return sv.lib().spec_expand_latent(desc(**d), x, w, ws, off, out, None)

    check(call, ["x", "w", "off", "out"], ["x", "w", "out"], [dict(ws=128 * 512 - 8), dict(ws=128 * 512 + 2)], [])
    assert sv.lib().spec_expand_latent(None, P, P, 65536, P, P, None) == NULL


def test_compaction():
    def call(B=2, wide=576, page=16, width=4, pages=9, **more):
        a = dict(pool=P, bt=P, ctx=P, off=P, parent=P, stop=P, new=None)
        a.update(more)
        return sv.lib().spec_compact_latent(B, wide, page, width, pages, *a.values(), None)

    for missing in ("pool", "bt", "ctx", "off", "stop"):
        assert call(**{missing: None}) == NULL, missing
    for bad in (dict(B=-1), dict(wide=0), dict(wide=-8), dict(wide=572), dict(width=-1), dict(pages=-1), dict(pool=P + 8)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(wide=584), dict(page=32), dict(B=65536)):
        assert call(**bad) == UNSUPPORTED, bad
    assert call(B=0) == 0


# ---- the binding ----
class _Stream:
    cuda_stream, device_index = 0, -1


def calls():
    """name -> (call with some arguments replaced, its good arguments); host tensors: refused at last for where they lie."""
    torch = pytest.importorskip("torch")
    b16 = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    f32 = lambda *s: torch.zeros(s)
    d = sv.make_latent_desc(**OK)
    places = dict(block_table=i32(2, 10), ctx_len=i32(2), q_offsets=i32(3), parent=None)
    return {
        "append": (sv.spec_append_latent, dict(latent=b16(8, 512), key=b16(8, 64), norm_weight=b16(512), inv_freq=f32(32), pool=b16(30, 16, 576), **places,
                                               positions=i32(8)), d),
        "absorb": (sv.spec_absorb_latent, dict(q=b16(8, 8, 192), w_key=b16(8, 128, 512), inv_freq=f32(32), ctx_len=i32(2), q_offsets=i32(3), parent=i32(8),
                                               q_out=b16(8, 8, 576), positions=i32(8)), d),
        "attend": (sv.spec_verify_attn_latent, dict(q=b16(8, 8, 576), pool=b16(30, 16, 576), **places, out=b16(8, 8, 512), lse=f32(8, 8),
                                                    workspace=torch.zeros(1 << 26, dtype=torch.uint8)), d),
        "expand": (sv.spec_expand_latent, dict(x=b16(8, 8, 512), w_value=b16(8, 128, 512), q_offsets=i32(3), out=b16(8, 8, 128)), d),
        "compact": (sv.spec_compact_latent, dict(pool=b16(30, 16, 576), **places, stop_node=i32(2), new_len=i32(2)), None),
    }


@pytest.mark.parametrize("name", ["append", "absorb", "attend", "expand", "compact"])
def test_binding_refuses_types_sizes_strides_and_host_memory(name):
    torch = pytest.importorskip("torch")
    fn, good, d = calls()[name]
    call = lambda **bad: fn(*([d] if d is not None else []), **{**good, **bad}, stream=_Stream())
    with pytest.raises(ValueError, match="device"):
        call()
    for key, t in good.items():
        if t is None or key == "workspace":
            continue
        with pytest.raises((TypeError, AssertionError)):
            call(**{key: t.double() if t.is_floating_point() else t.long()})
        smaller = t[:-1] if t.dim() == 1 else t[:, :-1]
        if not (name == "compact" and key in ("block_table", "ctx_len", "pool")):              # (what the sizes are taken from)
            with pytest.raises((ValueError, AssertionError)):
                call(**{key: smaller.contiguous()})
        apart = torch.zeros(t.shape + (2,), dtype=t.dtype)[..., 0]
        with pytest.raises((ValueError, AssertionError)):
            call(**{key: apart})
