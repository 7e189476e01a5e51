"""Counts of which the call has fewer rows (a batch of fixed size whose requests have more new tokens than it holds): appending and
attention take the same tokens of a request to be there, at the same places."""
import numpy as np
import pytest

import paged_ref as R
from paged_util import Cache, host, ints, randn
from paper_2601_20655_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("requests", [2, 70])
@pytest.mark.parametrize("past", [13, 40, 2 ** 31 - 1])
def test_new_tokens_behind_the_rows(requests, past):
    """12 rows; the last request with a token has them to q_start = `past`: it is as if it had them to 12."""
    import torch

    D, lens = 64, [64, 100] + [3] * (requests - 2)
    starts = [0, 4] + [past] * (requests - 1)
    k, v, q = (randn(i, (12, 1, D), "bf16") for i in (1, 2, 3))
    got = []
    for s in (starts, np.minimum(starts, 12)):
        c = Cache(lens, 1, D, 16, "bf16", "head", 3)
        args = list(c.args([4, 8] + [0] * (requests - 2)))
        args[3] = ints(s)
        B.dit_kv_append_forward(k, v, *args)
        for i in range(12):
            r, place = (0, lens[0] - 4 + i) if i < 4 else (1, lens[1] - 12 + i)
            page = int(c.table[r, place // 16])
            assert torch.equal(c.k[page, place % 16], k[i]) and torch.equal(c.v[page, place % 16], v[i]), i
        got.append((c, B.dit_attn_paged_forward(q, *args, frame=1)))
    assert torch.equal(got[0][0].k, got[1][0].k) and torch.equal(got[0][0].v, got[1][0].v)
    assert torch.equal(got[0][1], got[1][1])
    c = got[0][0]
    ref = R.attend(host(q), host(c.k), host(c.v), c.table, [0, 4, 12] + [12] * (requests - 2), lens, 1, 0, None, R.HALF["bf16"])
    R.check_attn(host(got[0][1]), None, ref, "bf16")
