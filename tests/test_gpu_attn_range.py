"""Attention over the paged cache at the ends of its arguments' ranges.  The tolerances are those of
the attention tests."""
import pytest
import test_gpu_attn as attn

pytestmark = pytest.mark.gpu

lc = attn.lc

FEW = [(7, 4), (3, 0), (1, 1), (5, 140)]
CHUNKS = [(90, 70), (150, 0), (1, 5), (100, 300)]


@pytest.mark.parametrize("window", [2**31 - 1, 2**31 - 3, 2**30, 2**30 - 1])
@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("seqs", [FEW, CHUNKS, [(90, 70)]])
def test_windows_longer_than_any_table(lc, seqs, fp8, window):
    """They hide nothing, where there are more new tokens than cached ones too."""
    c = attn.Case(seqs, 4, 2, 64, 16, fp8, seed=30)
    out, lse = c.call(lc, window=window)
    c.check(out, lse)
    want = c.call(lc)
    assert out.equal(want[0]) and lse.equal(want[1])
