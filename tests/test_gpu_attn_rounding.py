"""Roundings of the attention that the bounds of the other tests are too wide to see: to the nearest,
not towards zero, of the probabilities and of the output."""
import numpy as np
import pytest
import test_gpu_attn as attn

pytestmark = pytest.mark.gpu

lc = attn.lc


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("seqs", [[(1, 700), (1, 300)], [(90, 700), (1, 333)], [(1, 5000)]])
def test_probabilities_go_both_ways(lc, seqs, fp8):
    """Values of one: the rounded probabilities' sum over the sum of the unrounded ones.  Rounded to
    the nearest their errors cancel, and the quotient is 1 in bf16; cut off they would lower it by
    2^-9 to 2^-8, and the bf16 below 1 is 1 - 2^-8.  Of the rows that see 256 tokens and more: the
    errors are of deviation 2^-9 / sqrt(3) of a probability, and 2^-9 is 1.7 sqrt(1 / sum p^2) of
    the sum's, over 9 for the 30 or more tokens among which such a row's weight is spread."""
    c = attn.Case(seqs, 8, 2, 64, 16, fp8, seed=40, stale="")
    c.data[1] = 56 if fp8 else 1.0                # (1.0 in e4m3)
    if fp8:
        c.scales[1] = 127
    c.q *= 0.5                                     # no row hangs on a few tokens
    out, _ = c.call(lc)
    for b, (n, length) in enumerate(seqs):
        first = max(0, 255 - (length - n))
        if first < n:
            assert (out[c.starts[b] + first:c.starts[b] + n] == 1).all(), b


@pytest.mark.parametrize("n,length", [(1, 2), (40, 2)])
def test_output_to_the_nearest(lc, n, length):
    """Two tokens with the same key: half of each, a sum that is exact before it is rounded to bf16."""
    import torch
    c = attn.Case([(n, length)], 4, 2, 128, 16, False, seed=41, stale="")
    c.data[0] = 0.25
    out, lse = c.call(lc, causal=False)
    v = c.data[1, int(c.table[0, 0]), :, :2].double()                   # heads x 2 x D
    mean = (v[:, 0] + v[:, 1]) / 2
    nearest = (mean.float().to(torch.bfloat16).double() - mean).abs()
    for h in range(4):
        # (at a tie the sum's last bit in 32 decides)
        assert ((out[:, h].double() - mean[h // 2]).abs() <= nearest[h // 2] + 2.0 ** -20 * mean[h // 2].abs()).all()
    assert np.isfinite(lse.cpu().numpy()).all()
