"""Rows of more heads than a launch has wavefronts for are refused before anything is launched (the pointers are fake)."""
import pytest

from paper_2601_20655_amd import binding as B
from test_paged_host import UNSUPPORTED, append, rope

MOST = 2 ** 27


@pytest.mark.parametrize("H,Hk", [(MOST, 1), (1, MOST), (MOST // 2 + 1, MOST // 2), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("norm", [0, 1, 2])
def test_too_many_heads(H, Hk, norm):
    assert rope(N=1, H=H, Hk=Hk, norm=B.dit_qk_norm(norm, 1e-6, None, None)) == UNSUPPORTED


def test_too_many_heads_to_pages():
    assert append(N=1, H=MOST) == UNSUPPORTED
    assert append(N=1, H=2 ** 31 - 1) == UNSUPPORTED
    assert append(N=1, H=MOST - 2 ** 21, Hk=2 ** 20 + 1, n_pages=1, page_size=1) == UNSUPPORTED
