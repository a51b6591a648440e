"""Attention over the paged cache at the ends of its arguments' ranges.  The tolerances are those of
the attention tests."""
import numpy as np
import pytest
import test_gpu_attn as attn

from oracle import serve

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


def _whole_numbers(seqs, fp8, q0, k0, qi, ki, seed):
    """A case whose scores are exact in 32 bits: q and k are q0 and k0 in the first element and whole
    numbers from -3 to 3 times qi and ki in the others."""
    import torch
    c = attn.Case(seqs, 4, 2, 64, 16, fp8, seed=seed)
    rng = np.random.default_rng(seed)
    k = rng.integers(-3, 4, c.kv[0].shape) * float(ki)
    k[..., 0] = k0
    if fp8:
        codes, scales = serve.kv_encode(k)
        assert np.array_equal(serve.kv_decode(codes, scales), k)
        c.data[0], c.scales[0] = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    else:
        c.data[0] = torch.from_numpy(k).to(torch.bfloat16).cuda()
    c.kv[0] = k
    q = rng.integers(-3, 4, c.q.shape) * float(qi)
    q[..., 0] = q0
    c.q = torch.from_numpy(q).to(torch.bfloat16).cuda()
    return c


SEQS = [[(1, 300), (2, 45)], [(90, 200), (1, 130)], [(1, 3000)], [(40, 1500)]]


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("seqs", SEQS)
@pytest.mark.parametrize("e", [105, 127])
def test_scores_far_below_zero(lc, seqs, e, fp8):
    """q.k about -2^105 or -2^127 in every row, scaled to -256 and some tens around it."""
    c = _whole_numbers(seqs, fp8, 2.0 ** (e // 2 + 1), -2.0 ** (e - e // 2 - 1), 2.0 ** (e // 2 - 5), 2.0 ** (e - e // 2 - 5), 31)
    out, lse = c.call(lc, scale=2.0 ** (8 - e))
    c.check(out, lse, scale=2.0 ** (8 - e))


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("seqs", SEQS)
@pytest.mark.parametrize("common,scale", [(1024, 1.0), (1024, 0.03), (1024, 1e6), (64, 1e6), (0, 7e5), (0, 1e-30)])
def test_large_scaled_scores(lc, seqs, common, scale, fp8):
    """Scores of up to 10^12: what counts is by how much they differ."""
    c = _whole_numbers(seqs, fp8, common, common, 1, 1, 32)
    out, lse = c.call(lc, scale=scale)
    c.check(out, lse, scale=scale)


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("seqs", [[(1, 300), (2, 45)], [(1, 3000)], [(3, 2000)]])
def test_large_scores_of_one_row_leave_the_others_bits(lc, seqs, fp8):
    """Few rows: one query a hundred thousand times larger than those beside it."""
    c = attn.Case(seqs, 4, 2, 64, 16, fp8, seed=35)
    want = c.call(lc)
    c.q[0, 1] *= 1e5
    out, lse = c.call(lc)
    keep = [(t, h) for t in range(c.q.shape[0]) for h in range(4) if (t, h) != (0, 1)]
    for t, h in keep:
        assert out[t, h].equal(want[0][t, h]) and lse[t, h].equal(want[1][t, h]), (t, h)


@pytest.mark.parametrize("byte", [247, 254, 255])
@pytest.mark.parametrize("seqs", [[(4, 160), (1, 40)], [(90, 220), (1, 40)], [(90, 220)], [(150, 1500)]])
@pytest.mark.parametrize("window,back", [(0, 2), (0, 45), (50, 45), (50, 51), (50, 100)])
@pytest.mark.parametrize("keys", [False, True])
def test_scale_bytes_that_the_format_has_not(lc, keys, seqs, window, back, byte):
    """... of a token that some rows see (`back` before the last): the others are as without it,
    to the bit where it is the value's and their scores and maxima are the same."""
    c = attn.Case(seqs, 4, 2, 128, 16, True, seed=33)
    n, length = seqs[0]
    t = length - 1 - back
    clean = c.call(lc, window=window)
    c.scales[0 if keys else 1, c.table[0, t // 16], :, t % 16] = byte
    out, lse = c.call(lc, window=window)
    blind = [i for i in range(n) if not (t <= length - n + i and (window == 0 or t > length - n + i - window))]
    rows = blind + list(range(n, c.q.shape[0]))
    if not keys:
        for i in rows:
            assert out[i].equal(clean[0][i]) and lse[i].equal(clean[1][i]), i
    out[[i for i in range(n) if i not in blind]] = clean[0][[i for i in range(n) if i not in blind]]
    lse[[i for i in range(n) if i not in blind]] = clean[1][[i for i in range(n) if i not in blind]]
    c.check(out, lse, window=window)


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("new,length,window", [(512, 8192, 0), (512, 8192, 4096), (6, 8192, 0), (1, 8192, 4096)])
def test_a_value_that_is_no_number_costs_little(lc, new, length, window, fp8):
    """One NaN, or nothing but NaN on the last page, beside none: within ten times and half a millisecond."""
    import torch
    c = attn.Case([(new, length)], 8, 2, 128, 64, fp8, seed=34, stale="")
    table, lens, starts = c.dev(c.table), c.dev([length]), c.dev(c.starts)

    def ms():
        times = []
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            lc.attn_paged(c.q, c.data, table, lens, starts, c.scales, window=window)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)
    plain = ms()
    t = length - 2
    c.data[1, c.table[0, t // 64], 0, t % 64, 5] = 255 if fp8 else float("nan")
    one = ms()
    c.data[1, c.table[0, (length - 1) // 64]] = 255 if fp8 else float("nan")
    if window:
        t = length - new - window + 1
        c.data[1, c.table[0, t // 64]] = 255 if fp8 else float("nan")
    many = ms()
    assert max(one, many) <= 10 * plain + 0.5, (plain, one, many)
