"""Rows of a single token with more heads than one launch took."""
import pytest

from paged_util import ints
from paper_2601_20655_amd import binding as B

pytestmark = pytest.mark.gpu


def test_more_heads_than_wavefronts_of_a_launch():
    """A token of 84,000,000 heads of 128 (21.5 GB): as by calls of a few million of them each."""
    import torch

    H, D = 84_000_000, 128
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GiB")
    q = torch.empty((1, H, D), dtype=torch.bfloat16, device="cuda")
    for h in range(0, H, 12_000_000):
        q[:, h:h + 12_000_000].normal_()
    pos = ints([[7, 300, 41]])
    out = torch.full((1, H, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    B.dit_qk_rope_forward(q, None, pos, (44, 42, 42), q_out=out, norm=("head", 1e-6, None, None))
    for h in range(0, H, 12_000_000):
        part = q[:, h:h + 12_000_000]
        want, _ = B.dit_qk_rope_forward(part, None, pos, (44, 42, 42), norm=("head", 1e-6, None, None))
        assert torch.equal(out[:, h:h + 12_000_000], want), h
