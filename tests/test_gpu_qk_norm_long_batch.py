"""Per-token normalisation of more rows than one launch of 2^32 work items takes (a wavefront a row): rows repeat, and so do
the results."""
import pytest

from paper_2601_20655_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("many", ["queries", "keys"])
def test_more_rows_than_a_launch_takes(many):
    import torch

    Bn, L, D = 4, 1 << 24, 64
    gen = torch.Generator(device="cuda").manual_seed(0)
    few = torch.randn((1, 64, 1, D), generator=gen, device="cuda").bfloat16()
    norm = ("token", 1e-6, torch.rand(D, generator=gen, device="cuda") + 0.5, None)
    long = few.expand(Bn * L // 64, 64, 1, D).reshape(Bn, L, 1, D)
    if many == "queries":
        k, v = (torch.randn((1, 5, 1, D), generator=gen, device="cuda").bfloat16() for _ in range(2))
        want = B.dit_cross_attn_forward(few, k, v, norm=norm)
        got = B.dit_cross_attn_forward(long, *(t.expand(Bn, 5, 1, D).contiguous() for t in (k, v)), norm=norm)
        assert (got.view(-1, 64, 1, D) == want).all().item()
    else:
        # bit for bit what the batch entries give in calls of their own, whose launches are short enough
        v = torch.randn((1, 64, 1, D), generator=gen, device="cuda").bfloat16()
        v = v.expand(Bn * L // 64, 64, 1, D).reshape(Bn, L, 1, D)
        q = torch.randn((Bn, 16, 1, D), generator=gen, device="cuda").bfloat16()
        got = B.dit_cross_attn_forward(q, long, v, norm=norm, out_dtype=torch.float32)
        assert torch.isfinite(got).all().item()
        for b in range(Bn):
            assert torch.equal(got[b:b + 1], B.dit_cross_attn_forward(q[b:b + 1], long[b:b + 1], v[b:b + 1], norm=norm, out_dtype=torch.float32))
