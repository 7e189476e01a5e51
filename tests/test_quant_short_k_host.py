"""Which kernel 8-bit projections of less than one step of K (128) run on: all of K is then the cut step."""
import pytest

from test_quant_host import kernel_of

# kernel as test_quant_host.kernel_of names it, M, N: each tile with whole and with cut pieces of features, and the few rows'
# kernel with two or three workgroups a compute unit.  (64 x 128 tiles, "42", take no projection so short.)
SHORT = [("11 any", 33, 4128), ("11 any", 4152, 33), ("21 any", 8195, 8), ("21 any", 8244, 9), ("22 any", 10906, 136),
         ("22 any", 10951, 129), ("34 any", 11001, 264), ("34 any", 10940, 259), ("44 any", 12374, 264), ("44 any", 12371, 258),
         ("54 any", 10994, 520), ("54 any", 10936, 521), ("64 tail", 13728, 528), ("64 tail rest", 13667, 521),
         ("big tail", 16344, 560), ("big tail rest", 16382, 527), ("few1/4", 1, 15360), ("few1/4", 1, 20480), ("few2/4", 16, 15360),
         ("few2/4", 16, 20480)]
LENGTHS = [1, 15, 16, 34, 64, 100, 127]


@pytest.mark.parametrize("kernel,M,N", SHORT)
def test_every_tile_has_a_short_shape(kernel, M, N):
    assert [kernel_of(M, N, K) for K in LENGTHS] == [kernel] * len(LENGTHS)
