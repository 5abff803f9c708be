"""Tensors that the cache operators take as they come: larger than the batch, flat, of one request; and those in host
memory, which they refuse."""
import pytest

torch = pytest.importorskip("torch")

import cache_util as U
import test_quant_sizes as S
from paper_2503_10325_amd import binding as sv

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sv.lib()


def step(c, pools, change=None):
    """Appending, attention, compaction; `change` gets the device copies first.  Results, results first rows only."""
    d = U.Device(c, quant=pools)
    if change:
        change(d)
    d.append()
    out, lse = d.attend(d.q_out[:c["rows"]])
    new_len = d.compact(torch.full((len(c["ctx"]),), 1, dtype=torch.int32, device="cuda")) if d.table.dim() == 2 else None
    torch.cuda.synchronize()
    return [d.q_out[:c["rows"]], out, lse, d.k_pool, d.v_pool, d.k_scale, d.v_scale], new_len


def longer(x, rows):
    return torch.cat([x, torch.full((rows, *x.shape[1:]), -9, dtype=x.dtype, device=x.device)])


def test_buffers_for_a_larger_batch():
    c = U.batch(111, ctx=[30, 11, 64], n=[5, 3, 9], heads=(4, 2), tree=True)
    pools = U.quant_pools(c)

    def change(d):
        d.offsets, d.parent, d.q_out = longer(d.offsets, 4), longer(d.parent, 7), longer(d.q_out, 5)

    (want, want_len), (got, got_len) = step(c, pools), step(c, pools, change)
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and torch.equal(got_len, want_len)


def test_flat_block_table():
    c = U.batch(112, ctx=[30, 11, 64], n=[5, 3, 9], heads=(4, 2))
    pools = U.quant_pools(c)

    def change(d):
        d.table = d.table.reshape(-1)

    (want, _), (got, _) = step(c, pools, lambda d: None), step(c, pools, change)
    assert all(torch.equal(x, y) for x, y in zip(got[:3], want[:3]))


def test_one_request_of_a_wider_table():
    c = U.batch(113, ctx=[30], n=[5], heads=(4, 2))
    pools = U.quant_pools(c)

    def change(d):
        d.table = torch.cat([d.table, torch.full((1, 9), -1, dtype=torch.int32, device="cuda")], 1)

    (want, want_len), (got, got_len) = step(c, pools), step(c, pools, change)
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and torch.equal(got_len, want_len)


NAMES = dict(append_bf16=["q", "k", "v", "inv_freq", "k_pool", "v_pool", "block_table", "ctx_len", "q_offsets", "parent", "q_out", "positions"],
             append_quant=["q", "k_pool", "v_pool", "k_scale", "v_scale", "block_table", "q_out"],
             attend=["q", "k_pool", "v_pool", "k_scale", "v_scale", "block_table", "ctx_len", "q_offsets", "parent", "out", "lse", "workspace"],
             compact=["k_pool", "v_pool", "k_scale", "v_scale", "block_table", "ctx_len", "q_offsets", "parent", "stop_node", "new_len"])


@pytest.mark.parametrize("call,name", [(call, name) for call, names in NAMES.items() for name in names])
def test_one_tensor_in_host_memory_is_refused(monkeypatch, call, name):
    """On the host, before anything is launched."""
    class Library:                                                        # nothing reaches the GPU, whatever the binding lets through
        def __getattr__(self, entry):
            return getattr(real, entry) if entry.endswith("size") else lambda *a: pytest.fail("launched")

    real = sv.lib()
    monkeypatch.setattr(sv, "_lib", Library())
    for entry in ("spec_append_kv", "spec_append_kv_quant", "spec_verify_attn_quant", "spec_compact_kv_quant"):
        def moved(*desc, stream=None, own=getattr(sv, entry), **tensors):
            own(*desc, **{k: x if k == name else x.cuda() for k, x in tensors.items()})
        monkeypatch.setattr(sv, entry, moved)
    run = dict(append_bf16=lambda: S.append("bf16"), append_quant=lambda: S.append("quant"), attend=S.attend, compact=S.compact)[call]
    with pytest.raises(ValueError, match="device|cache"):
        run()
