"""The 8-bit operators together, as examples/int8_block.py runs them, against the block on 16-bit weights.

An 8-bit operand is off by at most half a scale, uniformly: scale / sqrt(12), the scale being amax / 127, and amax about 4.5
standard deviations of a row of these lengths: 1.0 % of an operand's RMS, 1.5 % of a product's.  What reaches the stream
passes at most five such products one after the other (qkv with attention's weights and values, out, up, down), attention and
the GELU between them stretching errors by no more than 1.5, and the stream's own part, which is not in 8 bits at all, is the
larger half of it: 1.5 % x sqrt(5) x 1.5 = 5 % at most."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,grid", [(2, (1, 1, 1)), (2, (2, 5, 9)), (4, (3, 16, 20))])
@pytest.mark.parametrize("stream_f32", [False, True])
def test_block_in_8_bits(heads, grid, stream_f32):
    import torch

    import int8_block as ex

    w = ex.make_weights(heads)
    h, x = ex.make_rows(heads, grid)
    if stream_f32:
        h = h.float()
    q = ex.quantise_weights(w)
    first = None
    for _ in range(2):  # (the same bits again)
        h8, x8 = ex.block_8(h, x, q, grid)
        assert h8.dtype == h.dtype and x8.dtype == torch.bfloat16
        if first is not None:
            assert torch.equal(first[0], h8) and torch.equal(first[1], x8)
        first = h8, x8
    h16, x16 = ex.block_16(h, x, w, grid)
    got, want = h8.float() + x8.float(), h16.float() + x16.float()
    rel = ((got - want).square().mean() / want.square().mean()).sqrt().item()
    print("heads %d grid %s: %.4f" % (heads, grid, rel))
    assert rel < 0.05
