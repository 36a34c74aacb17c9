"""Attention over the paged cache when a device-side wait runs out: the bound is the workspace's, the call ends, says so and
leaves nothing behind."""
import pytest
import torch

import kv_util as ku
import paper_2506_22694_b200 as vt

pytestmark = pytest.mark.gpu
I32 = torch.int32


# one row a sequence (parts joined by the attention kernel) and more (a second launch), rings of one place and of many, tree rows behind
# the tokens (the producers meet to read the parents), results of one CTA and of many, pages that come by tensor copies and row by row
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d,Hq,Hk,page,S,n,Q,N", [(128, 8, 8, 16, 1, 6000, 1, 0), (128, 32, 8, 32, 5, 900, 1, 0), (64, 8, 8, 16, 40, 700, 1, 0), (128, 8, 4, 7, 3, 900, 1, 0),
                                                  (64, 16, 4, 32, 6, 1500, 8, 40), (128, 32, 8, 16, 2, 2000, 10, 200), (256, 16, 4, 16, 3, 1500, 1, 0),
                                                  (256, 8, 2, 16, 2, 1200, 16, 30), (96, 12, 12, 24, 4, 800, 4, 12), (128, 4, 4, 64, 3, 100, 4, 9)])
def test_an_expired_wait_is_reported_and_the_workspace_stays_usable(d, Hq, Hk, page, S, n, Q, N, e4m3):
    """With the bound set to 1 ns the first wait that is not satisfied at once gives up.  A result that it keeps from being whole is NaN
    (all of a row, and its lse), every other one is as always; the calls behind it, on the same workspace and the same places on chip, are right."""
    host = ku.Host(S, n + N, Hk, d, page, e4m3, seed=d + S)
    dev, lens = host.device(), torch.tensor([max(1, n - 61 * s) for s in range(S)], dtype=I32).cuda()
    q = ku.bf16((S * Q, Hq, d), 3).cuda()
    node = parent = None
    if N:
        parent, node = ku.tree(S, N, 4).cuda(), torch.randint(-1, N, (S * Q,), generator=ku.gen(N)).to(I32).cuda()
    ws = ku.attend_ws(S, Q, Hq, Hk, d)
    call = lambda: vt.vt_kv_attend(q, dev, host.pages_dev, lens, node, parent, ws=ws)
    good = call()
    assert ws.read_status() == (0, 0, 0)
    for _ in range(5):
        ws.set_wait_limit(1)
        out, lse = call()
        again = call()
        ws.set_wait_limit(0)
        after = [call() for _ in range(3)]
        st, flags, _ = ws.read_status()
        assert (st, flags) == (5, vt.VT_FLAG_TIMEOUT) or (n < 200 and st == flags == 0)       # (a short call's few waits may all be satisfied at once)
        for o, l in ((out, lse), again):
            lost = torch.isnan(l)
            assert torch.equal(torch.isnan(o).all(-1), lost) and torch.equal(torch.isnan(o).any(-1), lost)
            assert torch.equal(o[~lost], good[0][~lost]) and torch.equal(l[~lost], good[1][~lost])
            assert bool(lost.any()) or n < 200
        for o, l in after:
            assert torch.equal(o, good[0]) and torch.equal(l, good[1])
    assert ws.read_status() == (0, 0, 0)


def test_a_captured_call_reads_the_bound_when_it_runs():
    host = ku.Host(2, 3000, 2, 128, 16, False, seed=2)
    dev, lens, q = host.device(), torch.tensor([3000, 2500], dtype=I32).cuda(), ku.bf16((2, 8, 128), 3).cuda()
    ws = ku.attend_ws(2, 1, 8, 2, 128)
    out = (torch.empty((2, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 8), device="cuda"))
    good = [x.clone() for x in vt.vt_kv_attend(q, dev, host.pages_dev, lens, out=out, ws=ws)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vt.vt_kv_attend(q, dev, host.pages_dev, lens, out=out, ws=ws)
    for limit in (0, 1, 10 ** 9, 1, 0):
        ws.set_wait_limit(limit)
        graph.replay()
        assert ws.read_status()[0] == (5 if limit == 1 else 0)
        assert limit == 1 or all(torch.equal(x, y) for x, y in zip(out, good))
