"""Attention over latents at lengths where the reference has to be worked out on the device, in 64 bits; bounds as in test_gpu_attn_latent.py."""
import pytest

torch = pytest.importorskip("torch")

from paper_2503_10325_amd import binding as sv

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sv.lib()


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("C,rope", [(512, 64), (256, 32)])
@pytest.mark.parametrize("H", [16, 32, 64, 128])
def test_long_pieces(H, C, rope, f32):
    """More tiles in a piece than page ids are held at a time; the reference in 64 bits on the device."""
    B, W, pages = 48, C + rope, 512
    g = torch.Generator(device="cuda").manual_seed(35)
    some = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)
    ctx = torch.randint(5000, 16 * pages - 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    held = 700
    pool, q = some(held, 16, W), some(B, H, W)
    table = torch.randint(0, held, (B, pages), generator=g, device="cuda", dtype=torch.int32)      # (requests may share pages)
    offsets = torch.arange(B + 1, device="cuda", dtype=torch.int32)
    scale = 0.05
    desc = sv.make_latent_desc(B, H, C, rope, 128, 128, B, 1, pages, held, scale=scale, out_dtype=sv.SPEC_F32 if f32 else sv.SPEC_BF16)
    assert f" {H} query rows" in sv.spec_describe_attn_latent_plan(desc)
    out = torch.empty(B, H, C, device="cuda", dtype=torch.float32 if f32 else torch.bfloat16)
    lse = torch.empty(B, H, device="cuda")
    workspace = torch.full((sv.spec_verify_attn_latent_workspace_size(desc),), 0xff, dtype=torch.uint8, device="cuda")
    sv.spec_verify_attn_latent(desc, q, pool, table, ctx, offsets, None, out, lse, workspace)
    own, t = (2.0 ** -24, 0.0) if f32 else (2.0 ** -8, 2.0 ** -8)
    for b in range(B):
        L = int(ctx[b]) + 1
        k = pool[table[b].long()].view(-1, W)[:L].double()
        qb, v = q[b].double(), k[:, :C].contiguous()
        s = scale * (qb @ k.T)
        ref_lse = torch.logsumexp(s, -1)
        w = torch.exp(s - ref_lse[:, None])
        ref, size = w @ v, w @ v.abs()
        e = 2.0 ** -19 * (1 + scale * (qb.abs() @ k.T.abs()).amax(-1)) + 2.0 ** -28 * L
        bound = (t + e)[:, None] * size
        assert torch.all((out[b].double() - ref).abs() <= bound + own * (ref.abs() + bound)), b
        assert torch.all((lse[b].double() - ref_lse).abs() <= e + 2.0 ** -22 * ref_lse.abs()), b
