"""The cache's calls at the end of the range of places that a page table may span."""
import math

import pytest
import torch

import kv_util as ku
import paper_2506_22694_b200 as vt

pytestmark = pytest.mark.gpu
I32 = torch.int32


def test_attention_over_the_longest_sequence():
    """2^31 - 32 places, by a table that names one page of 87392 tokens 24573 times: what that page alone gives, each weight 24573 times."""
    page, times = 32 * 2731, 24573
    n = page * times
    assert 2 ** 31 - 64 < n < 2 ** 31
    k, v = ku.bf16((1, 1, page, 64), 1).cuda(), ku.bf16((1, 1, page, 64), 2).abs().cuda()
    q = ku.bf16((1, 2, 64), 3).cuda()
    ws = ku.attend_ws(1, 1, 2, 1, 64)
    pages = torch.zeros((1, times), dtype=I32, device="cuda")
    one, one_lse = vt.vt_kv_attend(q, (k, v), pages, torch.tensor([page], dtype=I32).cuda(), ws=ws)
    out, lse = vt.vt_kv_attend(q, (k, v), pages, torch.tensor([n], dtype=I32).cuda(), ws=ws)
    assert ws.read_status() == (0, 0, 0)
    # sums of positive terms: an accumulator sees a team's tiles, of 148 CTAs' equal shares with eight teams each, by at most four additions a tile, each
    # off by half a step, 2^-24; both sums of the quotient; and two roundings to bf16
    off = n / (148 * 8 * 32) * 4 * 2.0 ** -24 + 2.0 ** -18
    assert float((out.float() / one.float() - 1).abs().max()) <= 2 * off + 2.0 ** -7
    assert float((lse - one_lse - math.log(times)).abs().max()) <= off + 2.0 ** -18
