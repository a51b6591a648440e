"""Few rows per sequence over long tables, where the visible tokens are dealt out to blocks and
the pieces joined: every number of rows a block holds, both head sizes and formats, with few
units (many pieces in each) and with many.  The tolerances are those of the attention tests."""
import pytest
import test_gpu_attn as attn

pytestmark = pytest.mark.gpu

lc = attn.lc


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [1, 3, 6])
def test_few_units(lc, new, D, fp8):
    """One cached head: 16 pieces in the unit and more."""
    c = attn.Case([(new, 9001)], 8, 1, D, 64, fp8, seed=new + D)
    c.check(*c.call(lc), heads=[0, 5, 7])
    c = attn.Case([(new, 5000), (new, 3), (new, 0), (new, 4100)], 16, 2, D, 16, fp8, seed=new + D)
    c.check(*c.call(lc), heads=[0, 7, 8, 15])


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [1, 3, 6])
def test_many_units(lc, new, D, fp8):
    """More units than every 16th block."""
    seqs = [(new, 2600)] + [(new, 1 + 997 * i % 2500) for i in range(19)]
    c = attn.Case(seqs, 16, 2, D, 32, fp8, seed=new + D)
    c.check(*c.call(lc), heads=[0, 15])


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("new", [1, 3, 6])
def test_values_that_are_no_numbers(lc, new, fp8):
    attn.test_values_that_are_no_numbers(lc, [(new, 5000), (new, 200)], fp8, 0)
    attn.test_values_that_are_no_numbers(lc, [(new, 5000), (new, 200)], fp8, 1500)
