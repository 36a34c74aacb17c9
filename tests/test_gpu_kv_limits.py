"""The cache's calls at the end of the range of places that a page table may span."""
import ctypes
import math

import pytest
import torch

import kv_util as ku
import paper_2506_22694_b200 as vt
from test_kv_refusals import KV

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


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_path_that_the_page_table_cannot_hold_is_not_committed(e4m3):
    """Not in part, and it does not count: lengths never pass what the table holds."""
    host = ku.Host(4, 40, 2, 64, 10, e4m3, seed=2)
    lens, n_accept = torch.tensor([38, 38, 40, 37], dtype=I32).cuda(), torch.tensor([2, 3, 1, 3], dtype=I32).cuda()
    path = torch.tensor([[0, 1, 2, 3], [1, 2, 3, -1], [0, -1, -1, -1], [0, 1, 2, -1]], dtype=I32).cuda()
    ws = vt.Workspace(vt.VT_CTRL_BYTES)
    assert host.pages.shape[1] * host.page == 40
    assert vt.vt_kv_commit(host.device(), host.pages_dev, lens, path, n_accept, ws=ws).tolist() == [40, 38, 40, 40]
    assert host.same() and ws.read_status()[:2] == (2, vt.VT_FLAG_BAD_PAGE)
    assert vt.vt_kv_commit(host.dev, host.pages_dev, lens, path, n_accept, out=lens, ws=ws) is lens and lens.tolist() == [40, 38, 40, 40]


def test_a_path_at_the_end_of_the_longest_sequence():
    page, times = 32 * 2731, 24573
    k = ku.bf16((1, 1, page, 64), 1).cuda()
    v, pages, room = k.clone(), torch.zeros((1, times), dtype=I32, device="cuda"), page * times
    path, ws = torch.arange(100, dtype=I32, device="cuda")[None], vt.Workspace(vt.VT_CTRL_BYTES)
    for n, taken in ((31, 31), (32, 0), (100, 0)):
        n_accept, lens = torch.tensor([n], dtype=I32).cuda(), torch.tensor([room - 31], dtype=I32).cuda()
        assert vt.vt_kv_commit((k, v), pages, lens, path, n_accept, ws=ws).tolist() == [room - 31 + taken]
        assert ws.read_status()[1] == (0 if taken else vt.VT_FLAG_BAD_PAGE)


def test_a_cache_that_no_tensor_map_describes_leaves_the_next_call_alone():
    """A stride of 2^40 bytes (of one page, never stepped over) is refused on the host, between two calls of another shape."""
    host = ku.Host(2, 100, 2, 64, 16, False, seed=3)
    dev, lens, q = host.device(), torch.tensor([100, 61], dtype=I32).cuda(), ku.bf16((2, 4, 64), 5).cuda()
    ws = ku.attend_ws(2, 1, 4, 2, 64)
    good = vt.vt_kv_attend(q, dev, host.pages_dev, lens, ws=ws)
    wide = KV(k=dev[0].data_ptr(), v=dev[1].data_ptr(), k_exp=None, v_exp=None, format=0, n_pages=1, heads=2, page=16, d=64, stride_page=2 ** 39,
              stride_head=16 * 64, stride_token=64, pages=host.pages_dev.data_ptr(), S=2, max_pages=host.pages.shape[1], pages_ld=host.pages.shape[1])
    out = torch.empty_like(good[0])
    stream = torch.cuda.current_stream().cuda_stream
    assert vt.lib().vt_kv_attend(q.data_ptr(), 256, 1, 4, ctypes.byref(wide), lens.data_ptr(), None, None, 0, 0, 0.125, out.data_ptr(), None, ws.ptr, ws.nbytes,
                                 stream) != vt.VT_OK
    got = vt.vt_kv_attend(q, dev, host.pages_dev, lens, ws=ws)
    assert torch.equal(got[0], good[0]) and torch.equal(got[1], good[1]) and ws.read_status() == (0, 0, 0)
