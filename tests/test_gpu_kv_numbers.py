"""Attention over the paged cache where numbers go to their ends: infinite queries beside missing tokens."""
import math

import pytest
import torch

import kv_util as ku
import paper_2506_22694_b200 as vt
from test_gpu_kv_attend import check

pytestmark = pytest.mark.gpu
I32 = torch.int32


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d,Hq,page", [(64, 4, 16), (64, 32, 16), (128, 24, 32), (128, 4, 7), (256, 2, 16), (256, 20, 16)])
def test_an_infinite_query_is_not_multiplied_with_what_is_missing(d, Hq, page, e4m3):
    """Its scores with the tokens that are there are all -inf: they weigh nothing, and the row has zeros.  The tiles are
    filled up behind the last token and in place of pages out of range, and infinity times such a zero is a NaN."""
    lens = [1, 17, 32, 45, 77, 160]
    host = ku.Host(len(lens), 160, 1, d, page, e4m3, seed=5)
    first = host.k.view(torch.uint8)[..., 0] if e4m3 else host.k[..., 0]
    first.copy_(torch.full_like(first, 0x38) if e4m3 else torch.ones_like(first))          # (0x38: one)
    q = ku.bf16((len(lens), Hq, d), 3)
    q[:, ::2, 0] = -math.inf
    check(host, q, lens, 1)
    broken = host.pages.clone()
    broken[5, 1] = -1
    ws = ku.attend_ws(len(lens), 1, Hq, 1, d)
    out, lse = vt.vt_kv_attend(q.cuda(), host.dev, broken.cuda(), torch.tensor(lens, dtype=I32).cuda(), ws=ws)
    assert bool((out[:, ::2] == 0).all()) and bool((lse[:, ::2] == -math.inf).all())
    assert bool(torch.isfinite(out.float()).all()) and bool(torch.isfinite(lse[:, 1::2]).all())
    assert ws.read_status()[1] == vt.VT_FLAG_BAD_PAGE
    node = torch.tensor([2, 0, -1, 1, 2, -1], dtype=I32)                                   # chains of up to three behind the committed tokens
    host = ku.Host(len(lens), 170, 1, d, page, e4m3, seed=6)
    first = host.k.view(torch.uint8)[..., 0] if e4m3 else host.k[..., 0]
    first.copy_(torch.full_like(first, 0x38) if e4m3 else torch.ones_like(first))
    check(host, q, lens, 1, node)
