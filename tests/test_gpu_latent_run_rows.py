"""A step of the latent operators in the attention kernels of 32, 64 and 128 query rows: against the model's own attention, in captured graphs that share a
workspace, on two streams, in pools whose offsets pass 32 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import latent_util as U
from latent_rows import Device
from oracle import latent as R

pytestmark = [pytest.mark.gpu, pytest.mark.parametrize("at_a_time", [32, 64, 128])]


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_10325_amd import binding
    binding.lib()


def step(d, stream=None):
    d.append(stream=stream)
    ql = d.absorb(stream=stream)
    o, _ = d.attend(ql, stream=stream)
    return d.expand(o, stream=stream)


@pytest.mark.parametrize("C,rope,nope,value", [(512, 64, 128, 128), (256, 32, 64, 64)])
@pytest.mark.parametrize("shape", [dict(ctx=[100, 33, 0], n=[3, 5, 7], H=24), dict(ctx=[40, 161], n=[20, 29], H=6, tree=True)])
def test_a_step_is_the_models_attention(at_a_time, shape, C, rope, nope, value):
    """Bounds as in test_gpu_latent_run.py: results of the attention are off by (2^-8 + e) sum w |c| and their rounding, within 2^-6.9 of what the product weighs
    them with; a query element by 2^-8, so a score by 2^-8 A and a weight by exp(2 2^-8 A) at most."""
    c = U.batch(61, **shape, C=C, rope=rope, nope=nope, value=value, interleaved=True, spread=0.0)
    c["q"] = U.bf16(c["q"] * 0.1)
    d = Device(c, at_a_time)
    got = U.host(step(d))
    pool, ql = U.host(d.pool), U.host(d.q_out)
    o, _, size, A, _ = R.attend(c, ql, pool, C, c["softmax"])
    want, size = R.expand(o, c["w_value"]), R.expand(size, np.abs(c["w_value"]))
    bound = 2.0 ** -6.9 * size
    assert np.all(np.abs(got - want) <= U.HALF * np.abs(want) + bound)
    model = R.model(c, c["q"], pool, c["w_key"], c["w_value"], c["softmax"])
    change = np.expm1(2.0 * 2.0 ** -8 * A)[..., None] * size
    assert np.all(np.abs(got - model) <= U.HALF * (np.abs(model) + change) + bound + change)


@pytest.mark.parametrize("f32", [False, True])
def test_captured_and_replayed(at_a_time, f32):
    """Two graphs that share a workspace, replayed with eager calls, other lengths and other queries between."""
    a = Device(U.batch(62, ctx=[900, 64], n=[9, 12], H=16), at_a_time, f32=f32)
    b = Device(U.batch(63, ctx=[2000, 0, 9], n=[12, 1, 4], H=40, tree=True, C=256, rope=32), at_a_time, f32=f32)
    shared = torch.full((max(a.workspace.numel(), b.workspace.numel()),), 0xff, dtype=torch.uint8, device="cuda")
    a.workspace = b.workspace = shared

    def run(d):
        d.append()
        return d.attend(d.absorb())

    run(a), run(b)
    torch.cuda.synchronize()
    graphs = []
    for d in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(d)
        graphs.append(g)
    for turn in range(4):
        for d, g in ((a, graphs[0]), (b, graphs[1])):
            d.ctx.copy_(torch.from_numpy(d.c["ctx"] - (turn * 37) % (d.c["ctx"].clip(1))))
            d.q.normal_()
            want, want_lse = (x.clone() for x in run(d))
            d.o.fill_(7.0)
            d.lse.fill_(7.0)
            shared.fill_(turn)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(d.o, want) and torch.equal(d.lse, want_lse)


def test_two_streams(at_a_time):
    """Batches on two streams at once, each with a workspace of its own."""
    ds = [Device(U.batch(64 + i, ctx=[3000, 500], n=[8, 5], H=16 + 20 * i), at_a_time) for i in range(2)]
    want = [step(d).clone() for d in ds]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for d in ds:
            d.out.fill_(7.0)
            d.o.fill_(7.0)
        torch.cuda.synchronize()
        for d, s in zip(ds, streams):
            step(d, stream=s)
        torch.cuda.synchronize()
        for d, w in zip(ds, want):
            assert torch.equal(d.out, w)


def test_pools_whose_offsets_pass_32_bits(at_a_time):
    """Pages behind 2^31 elements (4.5 GB)."""
    c = U.batch(66, ctx=[130, 20], n=[9, 12], H=16, tree=True)
    far, held = 240000, c["held"]
    keep = c["pool"]
    there = np.where(c["table"] >= 0, far - 1 - c["table"], -1).astype(np.int32)
    d = Device(dict(c, table=there, held=far, pool=keep[:1]), at_a_time)
    d.pool = torch.zeros((far, 16, 576), dtype=torch.bfloat16, device="cuda")
    d.pool[far - held:] = torch.from_numpy(keep[::-1].copy()).cuda().bfloat16()
    e = Device(c, at_a_time)
    assert torch.equal(step(d), step(e)) and torch.equal(d.lse, e.lse)
    assert torch.equal(d.pool[far - held:].flip(0), e.pool) and not torch.any(d.pool[:far - held])
