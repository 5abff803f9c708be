"""The binding of the cache operators refuses tensors that are smaller than the descriptor says, before anything is launched."""
import os

import pytest

from paper_2503_10325_amd import binding as sv

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.skipif(not os.path.exists(sv.LIB_PATH), reason="libspecverify.so not built")

B, HQ, HKV, D, TOTAL, WIDTH, PAGES = 2, 8, 2, 128, 8, 10, 30


class _Stream:
    cuda_stream = device_index = 0


def t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def i32(*shape):
    return t(*shape, dtype=torch.int32)


def f32(*shape):
    return t(*shape, dtype=torch.float32)


def quant():
    return dict(k_pool=t(PAGES, HKV, D // 16, 16, 16, dtype=torch.uint8), v_pool=t(PAGES, HKV, D, 16, dtype=torch.uint8),
                k_scale=f32(PAGES, HKV), v_scale=f32(PAGES, HKV))


def places():
    return dict(block_table=i32(B, WIDTH), ctx_len=i32(B), q_offsets=i32(B + 1), parent=i32(TOTAL))


def append(kind, **given):
    pools = quant() if kind == "quant" else dict(k_pool=t(PAGES, HKV, 16, D), v_pool=t(PAGES, HKV, 16, D))
    a = dict(q=t(TOTAL, HQ, D), k=t(TOTAL, HKV, D), v=t(TOTAL, HKV, D), inv_freq=f32(32), **pools, **places(),
             q_out=t(TOTAL, HQ, D), positions=i32(TOTAL))
    a.update(given)
    desc = sv.make_append_desc(B, HQ, HKV, D, TOTAL, 4, WIDTH, PAGES, 64)
    (sv.spec_append_kv_quant if kind == "quant" else sv.spec_append_kv)(desc, **a, stream=_Stream())


def attend(out_dtype=sv.SPEC_BF16, **given):
    out = f32 if out_dtype == sv.SPEC_F32 else t
    desc = sv.make_attn_desc(B, HQ, HKV, D, TOTAL, 4, WIDTH, out_dtype=out_dtype)
    a = dict(q=t(TOTAL, HQ, D), **quant(), **places(), out=out(TOTAL, HQ, D), lse=f32(TOTAL, HQ),
             workspace=t(sv.spec_verify_attn_quant_workspace_size(desc), dtype=torch.uint8))
    a.update(given)
    sv.spec_verify_attn_quant(desc, **a, stream=_Stream())


def compact(**given):
    a = dict(**quant(), **places(), stop_node=i32(B), new_len=i32(B))
    a.update(given)
    sv.spec_compact_kv_quant(**a, stream=_Stream())


SHORT = dict(block_table=i32(B - 1, WIDTH), q_offsets=i32(B), ctx_len=i32(B - 1), parent=i32(TOTAL - 1))


@pytest.mark.parametrize("kind", ["bf16", "quant"])
@pytest.mark.parametrize("name,small", [*SHORT.items(), ("block_table", i32(B, WIDTH - 1)), ("block_table", i32(B, WIDTH + 1)),
                                        ("block_table", i32(B * WIDTH - 1)), ("inv_freq", f32(31)), ("positions", i32(TOTAL - 1)),
                                        ("q_out", t(TOTAL, HQ - 1, D)), ("q_out", t(TOTAL - 1, HQ, D)), ("q_out", t(TOTAL, HQ, D // 2))])
def test_append(kind, name, small):
    with pytest.raises(ValueError, match=name):
        append(kind, **{name: small})


@pytest.mark.parametrize("out_dtype", [sv.SPEC_BF16, sv.SPEC_F32])
@pytest.mark.parametrize("name,small", [*SHORT.items(), ("block_table", i32(B, WIDTH - 1)), ("block_table", i32(B, WIDTH + 1)),
                                        ("q", t(TOTAL, HQ - 1, D)), ("q", t(TOTAL - 1, HQ, D)), ("out", (TOTAL - 1, HQ, D)),
                                        ("out", (TOTAL, HQ, D - 1)), ("lse", f32(TOTAL, HQ - 1)), ("lse", f32(TOTAL - 1, HQ))])
def test_attention(name, small, out_dtype):
    if name == "out":
        small = (f32 if out_dtype == sv.SPEC_F32 else t)(*small)
    with pytest.raises(ValueError, match=name):
        attend(out_dtype, **{name: small})


@pytest.mark.parametrize("name,small", [("block_table", i32(B - 1, WIDTH)), ("q_offsets", i32(B)), ("stop_node", i32(B - 1)),
                                        ("new_len", i32(B - 1))])
def test_compaction(name, small):
    with pytest.raises(ValueError, match=name):
        compact(**{name: small})


def test_the_type_comes_first():
    """A tensor that is of another type and too small is one of another type."""
    for call in (lambda **a: append("bf16", **a), lambda **a: append("quant", **a), attend, compact):
        with pytest.raises(TypeError, match="q_offsets"):
            call(q_offsets=t(1, dtype=torch.int64))
        with pytest.raises(AssertionError, match="contiguous"):
            call(q_offsets=i32(2 * B + 2)[::2])
