"""The cache operators together, as a serving loop uses them: new tokens appended, attention over cache and drafts, acceptance, the accepted
path moved into place; eagerly, on other streams, captured and replayed, over pools of more than 4 GB."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import cache_util as U
from oracle import cache as R
from paper_2503_10325_amd import binding as sv
from test_gpu_attn_quant import values_bound

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sv.lib()


def roomy(c, tokens):
    """The batch with pages for that many tokens of each request."""
    width = (tokens + R.PAGE - 1) // R.PAGE
    c["table"] = c["rng"].permutation(len(c["ctx"]) * width).astype(np.int32).reshape(-1, width)
    c["held"] = c["table"].size
    return c


def greedy(c, d, seed, V=48):
    """accept_len, stop_node by random logits that agree with the drafts about half the time."""
    rng = np.random.default_rng(seed)
    B, total = len(c["ctx"]), c["total"]
    tokens = rng.integers(0, 2, total).astype(np.int32)
    logits = torch.from_numpy(rng.standard_normal((total + B, V)).astype(np.float32)).cuda()
    logits[:, :2] += 6.0
    most = int(c["n"].max())
    accept_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    out, stop = torch.zeros(B, most + 1, dtype=torch.int32, device="cuda"), torch.full((B,), -1, dtype=torch.int32, device="cuda")
    need = sv.spec_accept_greedy_workspace_size(B, total, V)
    ws = torch.zeros(max(need, 16), dtype=torch.uint8, device="cuda")
    sv.spec_accept_greedy(B, total, most, d.offsets, d.parent, torch.from_numpy(tokens).cuda(), logits, accept_len, out, stop, None, ws)
    return accept_len, stop


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("heads,D", [((8, 2), 128), ((4, 4), 64)])
def test_decoding_steps(heads, D, tree):
    """Prompts, then four steps of drafts; every operator against the reference for the cache as it found it."""
    B = 5
    c = roomy(U.batch(51, ctx=[0] * B, n=[37, 1, 16, 90, 50], heads=heads, D=D), 160)
    d = U.Device(c, quant=U.quant_pools(c))
    ctx = np.zeros(B, dtype=np.int32)
    moved = 0
    for step in range(5):
        if step:
            n = np.random.default_rng(step).integers(1, 9, B)
            new = U.batch(52 + step, ctx=ctx, n=n, heads=heads, D=D, tree=tree)
            new["table"], new["held"] = c["table"], c["held"]
            pools = (d.k_pool, d.v_pool, d.k_scale, d.v_scale)
            c, d = new, U.Device(new)
            d.k_pool, d.v_pool, d.k_scale, d.v_scale = pools
        before = [U.host(x) for x in (d.k_pool, d.v_pool, d.k_scale, d.v_scale)]
        d.append()
        _, k, v, ks, vs, truth = R.append_quant(c, *before)
        assert np.array_equal(U.host(d.v_pool), v) and np.array_equal(U.host(d.v_scale), vs) and np.array_equal(U.host(d.k_scale), ks)
        other = U.host(d.k_pool) != k
        for pg, h, slot in truth:
            other[pg, h, :, slot] = False
        assert not other.any()
        now = [U.host(x) for x in (d.k_pool, d.v_pool, d.k_scale, d.v_scale)]
        out, lse = d.attend(d.q_out) if step else (None, None)            # (a prompt's attention is another operator's work)
        if step:
            ref, ref_lse = R.attend(c, U.host(d.q_out).astype(np.float64), *now)
            assert U.attn_close(U.host(out), ref, values_bound(c, now), False)
            assert np.all(np.abs(U.host(lse) - ref_lse) <= 2.0 ** -19 * np.maximum(np.abs(ref_lse), 8.0))
            accept_len, stop = greedy(c, d, step)
            new_len = d.compact(stop)
            want = R.compact_quant(c, *now, U.host(stop))
            for got, w in zip((d.k_pool, d.v_pool, d.k_scale, d.v_scale, new_len), want):
                assert np.array_equal(U.host(got), w)
            assert np.array_equal(U.host(new_len) - ctx, U.host(accept_len))
            ctx = U.host(new_len)
            moved += int((ctx - c["ctx"]).sum())
        else:
            ctx = ctx + c["n"].astype(np.int32)
    assert moved > 5


def test_long_prompts():
    """More than 1024 pages of new tokens: queries go with keys and values, one workgroup for a page's heads."""
    c = U.batch(60, ctx=[9, 100], n=[9001, 8003], heads=(3, 1), D=64)
    pools = U.quant_pools(c)
    d = U.Device(c, fused=True, quant=pools)
    d.append()
    q, k, v, ks, vs, truth = R.append_quant(c, *pools)
    assert U.rotated_close(U.host(d.q_out), q, c["q"], c["rotary"], 2.0 ** -8)
    assert np.array_equal(U.host(d.v_scale), vs) and np.array_equal(U.host(d.v_pool), v) and np.array_equal(U.host(d.k_scale), ks)
    got = U.host(d.k_pool)
    other = got != k
    for (pg, h, slot), x in truth.items():
        step = R.e4m3_step(x / ks[pg, h]) * ks[pg, h]
        assert np.all(np.abs(R.E4M3[got[pg, h, :, slot].reshape(-1)] * ks[pg, h] - x) <= step / 2 + 2.0 ** -20 * np.abs(c["k"]).max())
        other[pg, h, :, slot] = False
    assert not other.any()


def test_bf16_cache_feeds_attention():
    """Appended keys and values of the bf16 cache are what spec_verify_attn reads: against attention over the rotated tokens."""
    c = U.batch(61, ctx=[37, 0, 16], n=[5, 9, 1], heads=(4, 2), tree=True)
    pools = [U.bf16(c["rng"].standard_normal((c["held"], 2, 16, 128))) for _ in range(2)]
    d = U.Device(c, bf16_pools=pools)
    d.append()
    desc = sv.make_attn_desc(3, 4, 2, 128, c["total"], 9, c["table"].shape[1])
    ws = torch.zeros(max(16, sv.spec_verify_attn_workspace_size(desc)), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(d.q_out)
    sv.spec_verify_attn(desc, d.q_out, d.k_pool, d.v_pool, d.table, d.ctx, d.offsets, d.parent, out, None, ws)
    q, k, v = U.host(d.q_out).astype(np.float64), U.host(d.k_pool).astype(np.float64), U.host(d.v_pool).astype(np.float64)
    got = U.host(out)
    for b in range(3):
        o, n, ctx = c["offsets"][b], c["n"][b], c["ctx"][b]
        up = R.chains(c["parent"][o:o + n], n)
        for j in range(n):
            pos = np.array(list(range(ctx)) + [ctx + a for a in sorted(up[j])])
            pg = c["table"][b, pos // 16]
            for h in range(4):
                s = k[pg, h // 2, pos % 16] @ q[o + j, h] / np.sqrt(128.0)
                p = np.exp(s - s.max())
                ref = (p / p.sum()) @ v[pg, h // 2, pos % 16]
                # weights rounded to bf16 at worst (2^-8, and their sum likewise), the result's own rounding
                assert np.all(np.abs(got[o + j, h] - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -7 * np.abs(v[pg, h // 2, pos % 16]).max())


class Step:
    """append, attention, compaction with fixed addresses; `load` sets the cache and the lengths of a seed."""

    def __init__(self, seeds, workspace=None, heads=(8, 2), n=6, B=7, top=900):
        self.c = [roomy(U.batch(s, ctx=np.random.default_rng(s).integers(0, top, B), n=[n] * B, heads=heads, tree=True), top + 16) for s in seeds]
        for c in self.c[1:]:
            c["held"] = self.c[0]["held"]
        self.d = U.Device(self.c[0], quant=U.quant_pools(self.c[0]))
        self.sets = []
        for s, c in zip(seeds, self.c):
            x = U.Device(c, quant=U.quant_pools(c))
            stop = torch.from_numpy(np.random.default_rng(s).integers(-1, n, B).astype(np.int32)).cuda()
            self.sets.append((x, stop))
        self.names = ("q", "k", "v", "table", "ctx", "parent", "k_pool", "v_pool", "k_scale", "v_scale")
        self.stop, self.new_len = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
        c, d = self.c[0], self.d
        self.desc = sv.make_attn_desc(B, *heads, 128, c["rows"], n, c["table"].shape[1])
        self.need = sv.spec_verify_attn_quant_workspace_size(self.desc)
        self.ws = torch.full((self.need,), 0xff, dtype=torch.uint8, device="cuda") if workspace is None else workspace
        self.out, self.lse = torch.zeros_like(d.q_out), torch.zeros(c["rows"], heads[0], device="cuda")

    def load(self, i):
        x, stop = self.sets[i]
        for name in self.names:
            getattr(self.d, name).copy_(getattr(x, name))
        self.stop.copy_(stop)

    def run(self, stream=None):
        d = self.d
        d.append(stream=stream)
        sv.spec_verify_attn_quant(self.desc, d.q_out, d.k_pool, d.v_pool, d.k_scale, d.v_scale, d.table, d.ctx, d.offsets, d.parent,
                                  self.out, self.lse, self.ws, stream)
        sv.spec_compact_kv_quant(d.k_pool, d.v_pool, d.k_scale, d.v_scale, d.table, d.ctx, d.offsets, d.parent, self.stop, self.new_len, stream)

    def results(self):
        d = self.d
        return [x.clone() for x in (d.q_out, d.k_pool, d.v_pool, d.k_scale, d.v_scale, self.out, self.lse, self.new_len)]

    def eager(self, i):
        self.load(i)
        self.run()
        return self.results()


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def capture(step):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step.run()
    return graph


def test_replays_match_eager_calls():
    """Other lengths and another cache in each replay, eager calls with the same workspace between them."""
    step = Step([71, 72, 73])
    want = [step.eager(i) for i in range(3)]
    graph = capture(step)
    for k, i in enumerate((0, 1, 2, 2, 0, 1)):
        step.load(i)
        graph.replay()
        torch.cuda.synchronize()
        assert same(step.results(), want[i]), k
        if k % 2:
            assert same(step.eager((i + 1) % 3), want[(i + 1) % 3]), k
            torch.cuda.synchronize()


def test_two_graphs_share_a_workspace():
    a = Step([74, 75])
    b = Step([76, 77], heads=(4, 4), n=9, B=3, top=2500)
    ws = torch.full((max(a.need, b.need),), 0xff, dtype=torch.uint8, device="cuda")
    a.ws = b.ws = ws
    want = [[s.eager(i) for i in range(2)] for s in (a, b)]
    graphs = [capture(s) for s in (a, b)]
    for i in (0, 1, 1, 0):
        a.load(i), b.load(i)
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert same(a.results(), want[0][i]) and same(b.results(), want[1][i])


def test_two_streams_at_once():
    """Two loops on streams of their own, each with its workspace, many calls in flight."""
    steps = [Step([78, 79]), Step([80, 81], heads=(4, 4), n=9, B=3, top=2500)]
    want = [[s.eager(i) for i in range(2)] for s in steps]
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    got = [[], []]
    for k in range(6):
        for j, (s, stream) in enumerate(zip(steps, streams)):
            with torch.cuda.stream(stream):
                s.load(k % 2)
                s.run(stream)
                got[j].append(s.results())
    torch.cuda.synchronize()
    for j in range(2):
        for k in range(6):
            assert same(got[j][k], want[j][k % 2]), (j, k)


def test_pools_beyond_four_gigabytes():
    """Pages whose offsets need more than 32 bits; the tokens' pages are the pool's first and last."""
    H, D = 4, 128
    pages = (1 << 32) // (H * 16 * D) + 300
    c = U.batch(82, ctx=[70, 33], n=[5, 9], heads=(8, H), tree=True)
    low, c["held"] = c["held"], pages
    small = dict(c, held=low)
    pools = U.quant_pools(small)
    far = lambda p: np.where(p < low // 2, p, pages - low + p)
    d = U.Device(small, quant=pools)
    want = U.Device(small, quant=pools)
    want.append()
    ref = [x.clone() for x in want.attend(want.q_out)]
    stop = torch.tensor([4, 6], dtype=torch.int32, device="cuda")
    ref_len = want.compact(stop)
    ids = torch.from_numpy(far(np.arange(low))).cuda()
    for name in ("k_pool", "v_pool", "k_scale", "v_scale"):
        x = getattr(d, name)
        big = torch.empty((pages,) + tuple(x.shape[1:]), dtype=x.dtype, device="cuda")
        big[ids] = x
        setattr(d, name, big)
    assert d.k_pool.numel() > 1 << 32
    d.table = torch.from_numpy(np.where(c["table"] >= 0, far(c["table"]), -1).astype(np.int32)).cuda()
    d.append_desc = sv.make_append_desc(2, 8, H, D, c["rows"], 9, c["table"].shape[1], pages, D, False)
    d.append()
    out = d.attend(d.q_out)
    assert same(out, ref)
    assert torch.equal(d.compact(stop), ref_len)
    for name in ("k_pool", "v_pool", "k_scale", "v_scale"):
        assert torch.equal(getattr(d, name)[ids], getattr(want, name))


def test_a_cache_on_another_device_is_refused():
    class Elsewhere:
        device_index, cuda_stream = 1, 0

    c = U.batch(83, ctx=[3], n=[2], heads=(2, 1))
    d = U.Device(c, quant=U.quant_pools(c))
    for call in (lambda: d.append(stream=Elsewhere()), lambda: d.attend(d.q, stream=Elsewhere()),
                 lambda: d.compact(torch.zeros(1, dtype=torch.int32, device="cuda"), Elsewhere())):
        with pytest.raises(ValueError, match="device"):
            call()
