"""A token's request found among nearly as many as 31 bits hold, most of them without a token."""
import pytest

from paper_2601_20655_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("requests", [2 ** 31 - 130, 2 ** 31 - 64, 2 ** 31 - 1])
def test_nearly_all_requests(requests):
    """Tokens of the first request, of one inside and of the last."""
    import torch

    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GiB")
    inside = requests // 3
    start = torch.zeros(requests + 1, dtype=torch.int32, device="cuda")
    start[1:inside + 1] = 2
    start[inside + 1:requests] = 3
    start[requests] = 5
    lens = torch.full((requests,), 3, dtype=torch.int32, device="cuda")
    table = torch.full((requests, 1), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[inside, 0], table[requests - 1, 0] = 2, 0, 1
    k, v = (torch.randn((5, 1, 64), device="cuda").bfloat16() for _ in range(2))
    kc, vc = (torch.zeros((3, 4, 1, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.dit_kv_append_forward(k, v, kc, vc, table, start, lens)
    for rows, cache in ((k, kc), (v, vc)):
        want = torch.zeros_like(cache)
        want[2, 1:3], want[0, 2], want[1, 1:3] = rows[:2], rows[2], rows[3:]
        assert torch.equal(cache, want)
