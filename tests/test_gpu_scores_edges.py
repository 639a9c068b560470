"""Scores where a list of candidates runs over: rows whose first part tells nothing of what is largest."""
import math

import pytest
import torch

import score_ref as ref
from test_gpu_logprobs import BF16, DEV, F16, F32, INF, _check_scores, _labels, _logits

pytestmark = pytest.mark.gpu


def _api():
    from paper_2608_13144_amd import api
    return api


def _late(T, C, dtype, seed):
    """Rows of every kind whose largest classes come late, stand in one run, or are many equal ones."""
    x, g = _logits(T, C, dtype, seed)
    j = torch.arange(C, device=DEV)
    first = torch.randint(0, C - 700, (T, 1), generator=g, device=DEV)
    allowed = (j >= first) & (j < first + 600)
    x[::8] = torch.linspace(-9, 9, C, device=DEV).to(dtype)             # rising
    x[1::8] = torch.linspace(9, -9, C, device=DEV).to(dtype)
    x[2::8] = torch.where(allowed, x, torch.full_like(x, -INF))[2::8]   # one run allowed
    x[3::8] = torch.where(j >= C - 700, x + 20, x)[3::8]                # large ones at the end
    x[4::8, C // 2:] = 30.0                                             # more equal ones than a list holds
    x[5::16] = -INF
    x[13::16, : C - 300] = math.nan                                     # (the rest has what is likely)
    x[6::8] = torch.where(j % 997 == 5, x + 15, torch.full_like(x, torch.finfo(dtype).min))[6::8]  # few allowed, far apart
    x[7::16] = ((x * 2).round() / 2 - 20)[7::16]                        # few values, below zero
    x[15::16] = (x.float() * 2.0 ** -23).to(dtype)[15::16]              # next to zero
    return x, g


@pytest.mark.parametrize("k", [1, 8, 9, 16, 17, 32, 64])
@pytest.mark.parametrize("T,C,dtype", [(2100, 16384, BF16), (2049, 8190, F32), (2051, 9001, F16), (6001, 20480, F16),  # waves
                                       (2100, 7001, BF16), (2049, 3500, F32),
                                       (801, 9001, F32), (70, 131072, BF16), (33, 50021, F16), (17, 1 << 20, BF16)])
def test_rows_whose_large_classes_come_late(T, C, dtype, k):
    x, g = _late(T, C, dtype, T + C + k)
    y = _labels(T, C, g)
    out = _api().logprobs(x, y, top=k)
    fine = ~x.isnan().any(1)
    part = _api().LogProbs(*[v[fine] for v in (out.logp, out.lse, out.entropy, out.top_index, out.top_logp)])
    for lo in range(0, int(fine.sum()), 2048):   # (float64 copies of 2048 rows at a time)
        r = slice(lo, lo + 2048)
        _check_scores(x[fine][r], y[fine][r], k, 1.0, _api().LogProbs(
            part.logp[r], part.lse[r], part.entropy[r], part.top_index[r], part.top_logp[r]))
    assert torch.equal(out.top_index[~fine], ref.top(x[~fine], k))


@pytest.mark.parametrize("k", [2, 8, 9, 20, 32, 33, 64])
@pytest.mark.parametrize("T,C,dtype", [(300, 65, F32), (300, 200, F32), (2100, 250, F32), (300, 500, BF16), (300, 511, F16), (2100, 2048, F16)])
def test_short_rows_of_many_equal_values(T, C, dtype, k):
    """Few distinct values, so that more reach the threshold than a list holds."""
    x, g = _logits(T, C, dtype, C + k)
    x[::3] = x[::3].sign()
    x[1::6] = 0.25
    x[4::6] = torch.where(torch.arange(C, device=DEV) % 23 == 4, x, torch.full_like(x, torch.finfo(dtype).min))[4::6]
    x[5::12] = (x * 2).round()[5::12] / 2 - 20
    x[11::12] = (x.float() * 2.0 ** -23).to(dtype)[11::12]
    y = _labels(T, C, g)
    _check_scores(x, y, k, 1.0, _api().logprobs(x, y, top=k))


def _least_time(x, k):
    """Of eight calls, in milliseconds."""
    api, times = _api(), []
    for turn in range(6):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(8):
            api.logprobs(x, top=k)
        end.record()
        end.synchronize()
        times.append(begin.elapsed_time(end))
    return min(times[1:])


@pytest.mark.parametrize("T,C,dtype", [(2100, 16384, BF16), (4096, 8000, F32), (1024, 131072, BF16), (32768, 500, BF16)])
def test_no_row_is_read_once_for_each_alternative(T, C, dtype):
    """However the values lie: a call takes what a dozen readings take, not 64 (4 to 11 times the scores alone; 60 to 100 when the
    row was read once for each)."""
    rising = torch.linspace(-9, 9, C, device=DEV).to(dtype).repeat(T, 1)
    masked = torch.where(torch.arange(C, device=DEV) % (C // 12) == 3, rising, torch.full_like(rising, torch.finfo(dtype).min))
    alone = _least_time(rising, 0)
    for name, x in (("rising", rising), ("equal", torch.zeros_like(rising)), ("masked", masked)):
        assert _least_time(x, 64) < 24 * alone, name


@pytest.mark.parametrize("T,C,dtype", [(6001, 10000, F32), (4096, 8000, F32), (6001, 20480, F16)])
def test_many_alternatives_of_long_rows_cost_little_more_than_few(T, C, dtype):
    """64 take 1.4 to 1.5 times what eight take (2.8 to 3.7 times where a wave ranked them)."""
    x = _logits(T, C, dtype, 1)[0]
    assert _least_time(x, 64) < 2.1 * _least_time(x, 8)


def test_heads_where_a_pass_ends():
    """2^20 classes go through 512 rows at a time: the rows on both sides of each end."""
    from test_gpu_head_logprobs import _case, _check
    x, W, bias, y = _case(1100, 24, 1 << 20, BF16, 3)
    out = _api().head_logprobs(x, W, bias, y)
    for r in (slice(506, 518), slice(1018, 1030), slice(1094, 1100)):
        _check(x[r], W, bias, y[r], 1.0, _api().LogProbs(out.logp[r], out.lse[r], out.entropy[r], None, None))
