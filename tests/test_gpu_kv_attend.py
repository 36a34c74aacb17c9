"""Attention over the paged cache (Algorithm 2's drafter forward) against the same sums in 64 bits."""
import math

import pytest
import torch

import kv_util as ku
import paper_2506_22694_b200 as vt

pytestmark = pytest.mark.gpu
I32 = torch.int32


def check(host, q, lens, Q, node=None, parent=None, scale=None, ws=None, flags=0):
    Hq = q.shape[1]
    ws = ws or ku.attend_ws(host.S, Q, Hq, host.heads, host.d)
    dev = host.device()
    out, lse = vt.vt_kv_attend(q.cuda(), dev, host.pages_dev, torch.tensor(lens, dtype=I32).cuda(), None if node is None else node.cuda(),
                               None if parent is None else parent.cuda(), scale, ws=ws)
    ref, ref_l, tol, tol_l = ku.attend(host, q, lens, Q, node, parent, scale)
    ok, worst = ku.near(out, ref, tol)
    assert ok, "out is %.3g of its bound off" % worst
    ok, worst = ku.near(lse, ref_l, tol_l)
    assert ok, "lse is %.3g of its bound off" % worst
    assert ws.read_status()[1] == flags
    return out, lse


def check_again(host, q, lens, Q, node, parent):
    dev = lambda x: None if x is None else x.cuda()
    return vt.vt_kv_attend(q.cuda(), host.dev, host.pages_dev, torch.tensor(lens, dtype=I32).cuda(), dev(node), dev(parent))


# one row a sequence: every head size and format, groups of query heads, page sizes that do and do not divide a tile, lengths around its edges
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d,Hq,Hk,page", [(64, 8, 8, 16), (64, 32, 8, 7), (96, 4, 4, 32), (128, 8, 8, 16), (128, 32, 8, 64), (128, 28, 4, 5),
                                          (192, 6, 2, 24), (256, 8, 1, 16), (128, 40, 2, 1)])
def test_single_tokens(d, Hq, Hk, page, e4m3):
    lens = [0, 1, 15, 16, 17, 63, 64, 65, 130, 257]
    host = ku.Host(len(lens), 260, Hk, d, page, e4m3, seed=d + page)
    check(host, ku.bf16((len(lens), Hq, d), 3, 1.5), lens, 1)


# rows of a tree: one to 64 rows a sequence, groups that fill one, two and four bands of 16 rows, and more than one group of four
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d,Hq,Hk,Q,N,page", [(64, 8, 8, 8, 24, 16), (128, 32, 8, 4, 13, 16), (128, 32, 8, 8, 72, 32), (128, 8, 8, 10, 200, 12),
                                              (128, 32, 8, 16, 40, 16), (128, 16, 8, 33, 50, 16), (96, 8, 4, 60, 90, 9), (192, 4, 2, 17, 20, 16),
                                              (256, 4, 2, 9, 30, 16), (256, 8, 2, 20, 33, 8), (128, 16, 4, 64, 130, 16)])
def test_tree_rows(d, Hq, Hk, Q, N, page, e4m3):
    lens = [0, 5, 70, 33]
    S = len(lens)
    host = ku.Host(S, 70 + N, Hk, d, page, e4m3, seed=d + Q)
    parent = ku.tree(S, N, Q)
    node = torch.randint(-2, N, (S * Q,), generator=ku.gen(N)).to(I32)
    check(host, ku.bf16((S * Q, Hq, d), 5, 1.2), lens, Q, node, parent)


@pytest.mark.parametrize("e4m3", [False, True])
def test_chains_need_no_parents(e4m3):
    host = ku.Host(3, 60, 2, 128, 16, e4m3, seed=9)
    node = torch.arange(12, dtype=I32).repeat(3)
    check(host, ku.bf16((36, 8, 128), 6), [0, 31, 40], 12, node, None)


def test_one_long_sequence_is_split_and_joined_the_same_way_every_time():
    for e4m3 in (False, True):
        for Hq, Hk, d, Q, N in ((8, 8, 128, 1, 0), (32, 8, 128, 2, 40), (8, 2, 64, 12, 70), (16, 2, 256, 8, 9)):
            host = ku.Host(1, 3100 + N, Hk, d, 16, e4m3, seed=N)
            node = torch.randint(0, N, (Q,), generator=ku.gen(1)).to(I32) if N else None
            q = ku.bf16((Q, Hq, d), 8, 1.5)
            ws = ku.attend_ws(1, Q, Hq, Hk, d)
            a = check(host, q, [3001], Q, node, ku.tree(1, N, 4) if N else None, ws=ws)
            for _ in range(3):
                b = check(host, q, [3001], Q, node, ku.tree(1, N, 4) if N else None, ws=ws)
                assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_many_sequences_of_very_different_lengths():
    lens = [(37 * i * i) % 401 if i % 7 else 0 for i in range(150)]       # (more sequences than a CTA has threads)
    host = ku.Host(150, 401, 2, 64, 16, False, seed=4)
    check(host, ku.bf16((150, 4, 64), 1), lens, 1)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d,Hq,Hk,Q,page", [(128, 4, 4, 1, 32), (128, 4, 4, 1, 16), (128, 8, 4, 8, 48), (64, 4, 4, 1, 96), (64, 16, 4, 8, 32), (256, 4, 4, 1, 64), (96, 4, 4, 1, 24)])
def test_enough_tokens_for_many_turns_of_every_place_on_chip(d, Hq, Hk, Q, page, e4m3):
    """About one whole result for each SM, every one of many rounds, and a tree behind each."""
    lens = [1500 + 23 * (i % 9) for i in range(37)]
    host = ku.Host(37, 1800, Hk, d, page, e4m3, seed=d + page)
    node = torch.randint(-1, 20, (37 * Q,), generator=ku.gen(5)).to(I32) if Q > 1 else None
    q = ku.bf16((37 * Q, Hq, d), 7, 1.5)
    a = check(host, q, lens, Q, node, ku.tree(37, 20, 3) if Q > 1 else None)
    for _ in range(3):
        b = check_again(host, q, lens, Q, node, ku.tree(37, 20, 3) if Q > 1 else None)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_more_sequences_than_lengths_are_kept_for():
    lens = [(7 * i) % 90 for i in range(1300)]
    host = ku.Host(1300, 90, 1, 64, 16, True, seed=4)
    check(host, ku.bf16((1300, 2, 64), 1), lens, 1)


def test_a_scale_of_its_own_strided_queries_and_other_layouts():
    for e4m3 in (False, True):
        for page in (16, 6):
            host = ku.Host(3, 50, 2, 128, page, e4m3, seed=2, layout="nphd")
            wide = ku.bf16((3, 5 * 8 * 128), 4)
            q = wide.view(3, 40, 128)[:, 8:16]
            for scale in (0.25, -0.1, 0.0):
                dev = host.device()
                got, lse = vt.vt_kv_attend(wide.cuda().view(3, 40, 128)[:, 8:16], dev, host.pages_dev, torch.tensor([50, 1, 17], dtype=I32).cuda(), scale=scale)
                ref, ref_l, tol, tol_l = ku.attend(host, q, [50, 1, 17], 1, scale=scale)
                assert ku.near(got, ref, tol)[0] and ku.near(lse, ref_l, tol_l)[0]


def test_what_lies_in_unseen_places_does_not_matter():
    """NaN and infinities behind the last token, in nodes of other branches and in pages of nobody."""
    for e4m3 in (False, True):
        for bad in (math.nan, math.inf, -math.inf):
            for Hq, Q in ((4, 3), (16, 3), (32, 4)):
                host = ku.Host(2, 60, 2, 64, 16, e4m3, seed=7)
                lens, N = [19, 32], 14
                parent = torch.tensor([[-1, -1, 0, 0, 1, 2, 2, 3, 4, 4, 5, 5, 6, 7]] * 2, dtype=I32)
                node = torch.tensor([10, 9, -1, 3][:Q] + [12, 4, -2, 0][:Q], dtype=I32)
                seen = {0: [set(), set()], 1: [set(), set()]}
                for s in range(2):
                    tokens = set(range(lens[s]))
                    for r in range(Q):
                        f = int(node[s * Q + r])
                        while f >= 0:
                            tokens.add(lens[s] + f)
                            f = int(parent[s, f])
                    seen[s] = {host.place(s, i) for i in tokens}
                keep = seen[0] | seen[1]
                for p in range(host.k.shape[0]):
                    for j in range(16):
                        if (p, j) in keep:
                            continue
                        if e4m3:
                            host.ke[p, :, j] = host.ve[p, :, j] = 255
                            host.k.view(torch.uint8)[p, :, j] = host.v.view(torch.uint8)[p, :, j] = 127
                        else:
                            host.k[p, :, j] = host.v[p, :, j] = bad
                q = ku.bf16((2 * Q, Hq, 64), 3)
                out, _ = check(host, q, lens, Q, node, parent)
                assert bool(torch.isfinite(out).all())


def test_a_node_that_is_no_number_reaches_only_the_rows_that_see_it():
    for e4m3 in (False, True):
        for what in ("v", "k"):
            for Hq, Q in ((4, 4), (16, 4), (32, 5)):
                host = ku.Host(1, 60, 2, 64, 16, e4m3, seed=11)
                parent = torch.tensor([[-1, -1, 0, 1, 2, 3]], dtype=I32)
                node = torch.tensor([4, 5, 2, 3, -1][:Q], dtype=I32)
                p, j = host.place(0, 21 + 0)                              # node 0: rows of nodes 4 and 2 see it
                if e4m3:
                    (host.ve if what == "v" else host.ke)[p, :, j] = 255
                else:
                    (host.v if what == "v" else host.k)[p, :, j, 5] = math.nan
                    if what == "v":
                        host.v[p, :, j, 40] = math.inf
                out, _ = check(host, ku.bf16((Q, Hq, 64), 3), [21], Q, node, parent)
                finite = torch.isfinite(out.float()).all(-1).all(-1).cpu().tolist()
                assert finite == [False, True, False, True, True][:Q]


def test_scores_without_a_bound():
    """Infinite scores: -inf weighs nothing, a row of nothing else has zeros, +inf is no number (inf - inf), as in the formula."""
    host = ku.Host(3, 20, 1, 64, 16, False, seed=1)
    for i in range(20):
        for s, value in ((1, -math.inf), (2, math.inf)):
            p, j = host.place(s, i)
            if i >= 10 or s == 1:
                host.k[p, :, j, 0] = value
    q = ku.bf16((3, 4, 64), 2).abs() + 0.5
    dev = host.device()
    out, lse = vt.vt_kv_attend(q.cuda(), dev, host.pages_dev, torch.tensor([20, 20, 20], dtype=I32).cuda())
    assert bool(torch.isfinite(out[0]).all())
    assert bool((out[1] == 0).all()) and bool((lse[1] == -math.inf).all())
    assert bool(torch.isnan(out[2]).all()) and bool(torch.isnan(lse[2]).all())


def test_large_scores_do_not_overflow():
    host = ku.Host(2, 90, 2, 128, 16, False, seed=3, std=30.0)
    check(host, ku.bf16((2, 8, 128), 2, 30.0), [90, 33], 1)


def test_pages_lengths_and_nodes_out_of_range_are_left_out_and_flagged():
    for page in (16, 10):
        host = ku.Host(2, 64, 2, 128, page, False, seed=5)
        q = ku.bf16((2, 4, 128), 2)
        ws = ku.attend_ws(2, 1, 4, 2, 128)
        room = host.pages.shape[1] * page
        check(host, q, [-5, 3], 1, ws=ws)                                 # a negative length is none
        broken = host.pages.clone()
        broken[0, 1], broken[1, 0] = host.k.shape[0], -1
        out, lse = vt.vt_kv_attend(q.cuda(), host.device(), broken.cuda(), torch.tensor([40, 2 * page], dtype=I32).cuda(), ws=ws)
        st, flags, _ = ws.read_status()
        assert flags == vt.VT_FLAG_BAD_PAGE and st == 2
        for s, seen in ((0, list(range(page)) + list(range(2 * page, 40))), (1, list(range(page, 2 * page)))):
            k, v = host.values(s, seen)
            for h in range(4):
                z = k[:, h // 2] @ q[s, h].double() * 128 ** -0.5
                assert abs(float(torch.logsumexp(z, 0)) - float(lse[s, h])) < 1e-4
                ref = torch.softmax(z, 0) @ v[:, h // 2]
                assert float((out[s, h].double().cpu() - ref).abs().max()) <= 2.0 ** -8 * float(ref.abs().max()) + 1e-4
        out, lse = vt.vt_kv_attend(q.cuda(), host.dev, host.pages_dev, torch.tensor([room + 1, 2 ** 31 - 1], dtype=I32).cuda(), ws=ws)
        same, _ = vt.vt_kv_attend(q.cuda(), host.dev, host.pages_dev, torch.tensor([room, room], dtype=I32).cuda(), ws=ws)
        assert torch.equal(out, same)
        ws.read_status()
        node = torch.tensor([9, 2 ** 31 - 1], dtype=I32).cuda()
        parent = torch.full((2, 9), -1, dtype=I32).cuda()
        out, _ = vt.vt_kv_attend(q.cuda(), host.dev, host.pages_dev, torch.tensor([30, 12], dtype=I32).cuda(), node, parent, ws=ws)
        assert ws.read_status()[1] == vt.VT_FLAG_BAD_PAGE
        same, _ = vt.vt_kv_attend(q.cuda(), host.dev, host.pages_dev, torch.tensor([30, 12], dtype=I32).cuda(), ws=ws)
        assert float((out.float() - same.float()).abs().max()) <= 2.0 ** -7 * float(same.float().abs().max())
        # nodes whose place the table does not reach
        node = torch.tensor([3, 0], dtype=I32).cuda()
        vt.vt_kv_attend(q.cuda(), host.dev, host.pages_dev, torch.tensor([room - 2, 12], dtype=I32).cuda(), node, parent, ws=ws)
        assert ws.read_status()[1] == vt.VT_FLAG_BAD_PAGE


def test_parents_that_do_not_lie_in_front_end_the_walk():
    host = ku.Host(1, 40, 1, 64, 16, False, seed=3)
    parent = torch.tensor([[0, 2, 1, 7, -9, 4]], dtype=I32)               # node 0: itself; 1: behind it; 3: behind it; 4: below -1
    node = torch.tensor([0, 1, 2, 3, 4, 5], dtype=I32)
    check(host, ku.bf16((6, 2, 64), 3), [10], 6, node, parent)


def test_the_largest_tree_and_a_chain_through_all_of_it():
    host = ku.Host(1, 2100, 1, 64, 16, False, seed=3)
    node = torch.tensor([2047, 5, 1000], dtype=I32)
    check(host, ku.bf16((3, 2, 64), 3), [40], 3, node, None)
    check(host, ku.bf16((3, 2, 64), 3), [40], 3, node, torch.arange(-1, 2047, dtype=I32)[None])


def test_offsets_beyond_32_bits():
    """A cache of 5 GB each for keys and values; the sequences' pages lie at both ends."""
    free, _ = torch.cuda.mem_get_info()
    if free < 14 << 30:
        pytest.skip("needs 14 GB")
    heads, page, d = 8, 64, 128
    n = 5 * 2 ** 30 // (heads * page * d * 2)
    host = ku.Host(2, 300, heads, d, page, False, seed=8)
    k, v = (torch.empty((n, heads, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    used = host.pages.flatten().tolist()
    there = [n - 1 - i if i % 2 else i for i in range(len(used))]
    pages = torch.tensor(there, dtype=I32).view(host.pages.shape).cuda()
    for a, b in zip(used, there):
        k[b], v[b] = host.k[a].cuda(), host.v[a].cuda()
    q = ku.bf16((2, 16, d), 4)
    out, lse = vt.vt_kv_attend(q.cuda(), (k, v), pages, torch.tensor([300, 129], dtype=I32).cuda())
    ref, ref_l, tol, tol_l = ku.attend(host, q, [300, 129], 1)
    assert ku.near(out, ref, tol)[0] and ku.near(lse, ref_l, tol_l)[0]
    x = ku.bf16((2, heads, d), 6)
    vt.vt_qkv_write(None, x.cuda(), (2 * x).cuda(), (k, v), pages, torch.tensor([299, 130], dtype=I32).cuda())
    rk, rv = vt.vt_kv_read((k, v), pages, torch.tensor([299, 130], dtype=I32).cuda())
    assert torch.equal(rk.cpu(), x) and torch.equal(rv.cpu(), 2 * x)
    path = torch.tensor([[3, -1, -1, -1], [2, -1, -1, -1]], dtype=I32).cuda()
    vt.vt_kv_commit((k, v), pages, torch.tensor([296, 128], dtype=I32).cuda(), path, torch.tensor([1, 1], dtype=I32).cuda())
    rk, _ = vt.vt_kv_read((k, v), pages, torch.tensor([296, 128], dtype=I32).cuda())
    assert torch.equal(rk.cpu(), x)


def test_a_captured_call_follows_the_lengths():
    host = ku.Host(3, 400, 2, 128, 16, False, seed=8)
    dev = host.device()
    q = ku.bf16((3, 8, 128), 4)
    qd, lens = q.cuda(), torch.tensor([1, 1, 1], dtype=I32).cuda()
    ws = ku.attend_ws(3, 1, 8, 2, 128)
    out = (torch.empty((3, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((3, 8), device="cuda"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        vt.vt_kv_attend(qd, dev, host.pages_dev, lens, out=out, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vt.vt_kv_attend(qd, dev, host.pages_dev, lens, out=out, ws=ws)
    for now in ([400, 0, 7], [16, 399, 200], [0, 0, 0], [400, 400, 400]):
        lens.copy_(torch.tensor(now, dtype=I32))
        graph.replay()
        ref, ref_l, tol, tol_l = ku.attend(host, q, now, 1)
        assert ku.near(out[0], ref, tol)[0] and ku.near(out[1], ref_l, tol_l)[0]


def test_two_streams_with_a_workspace_each():
    host = ku.Host(2, 300, 2, 128, 16, False, seed=8)
    dev = host.device()
    q = [ku.bf16((2, 8, 128), 4 + i).cuda() for i in range(2)]
    lens = torch.tensor([300, 77], dtype=I32).cuda()
    ref = [vt.vt_kv_attend(x, dev, host.pages_dev, lens)[0] for x in q]
    torch.cuda.synchronize()
    streams, spaces = [torch.cuda.Stream() for _ in range(2)], [ku.attend_ws(2, 1, 8, 2, 128) for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(vt.vt_kv_attend(q[i], dev, host.pages_dev, lens, ws=spaces[i])[0])
    torch.cuda.synchronize()
    assert all(torch.equal(x, ref[i]) for i in range(2) for x in got[i])


def test_no_sequences():
    host = ku.Host(1, 10, 2, 64, 16, False, seed=8)
    dev = host.device()
    out, lse = vt.vt_kv_attend(torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda"), dev, host.pages_dev[:0], torch.empty(0, dtype=I32, device="cuda"))
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)


@pytest.mark.parametrize("page_id", [-1, -2, -3, -2 ** 31, 2 ** 31 - 1])
def test_any_page_id_out_of_range_is_flagged(page_id):
    for e4m3 in (False, True):
        host = ku.Host(1, 40, 1, 64, 16, e4m3, seed=8)
        broken = host.pages.clone()
        broken[0, 1] = page_id
        q, ws = ku.bf16((1, 2, 64), 2), ku.attend_ws(1, 1, 2, 1, 64)
        out, _ = vt.vt_kv_attend(q.cuda(), host.device(), broken.cuda(), torch.tensor([32], dtype=I32).cuda(), ws=ws)
        assert ws.read_status()[1] == vt.VT_FLAG_BAD_PAGE
        ref, _, tol, _ = ku.attend(host, q, [16], 1)                      # (what the first page holds)
        ok, worst = ku.near(out, ref, tol)
        assert ok, worst


@pytest.mark.parametrize("power", [106, -106])
def test_powers_of_queries_and_keys_that_undo_each_other(power):
    """Keys of 2^113 (their sum with a query of 2^14 in f16 would not fit fp32) under queries of 2^-112, and the other way round."""
    for Hq in (2, 32):
        host = ku.Host(2, 70, 2, 64, 16, True, seed=4)
        host.ke = torch.full_like(host.ke, 127 + power)
        q = (ku.bf16((2, Hq, 64), 3).float() * 2.0 ** (-power - 6)).to(torch.bfloat16)
        check(host, q, [70, 9], 1)


@pytest.mark.parametrize("S", [31, 32, 33, 384, 385])
def test_sequences_about_the_numbers_at_which_they_are_dealt_out_otherwise(S):
    for Q in (1, 9):
        host = ku.Host(S, 40, 1, 64, 8, False, seed=S)
        lens = [(7 * s) % 41 for s in range(S)]
        lens[-1] = 0
        check(host, ku.bf16((S * Q, 2, 64), 6), lens, Q)


def test_two_captured_calls_share_a_workspace():
    """Their partial results lie in the same places: replays in turn, on one stream, are what the calls give by themselves."""
    a, b = ku.Host(1, 4000, 2, 64, 16, False, seed=1), ku.Host(3, 2500, 2, 64, 16, False, seed=2)
    ws = ku.attend_ws(3, 9, 4, 2, 64)
    calls = []
    for host, Q, lens in ((a, 1, [4000]), (b, 9, [2500, 0, 1700]), (b, 2, [31, 2222, 1])):
        q = ku.bf16((host.S * Q, 4, 64), Q).cuda()
        dev, n = host.device(), torch.tensor(lens, dtype=I32).cuda()
        out = (torch.empty_like(q), torch.empty(q.shape[:2], device="cuda"))
        call = lambda q=q, dev=dev, pages=host.pages_dev, n=n, out=out: vt.vt_kv_attend(q, dev, pages, n, out=out, ws=ws)
        call()
        torch.cuda.synchronize()
        want = [x.clone() for x in out]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        calls.append((graph, out, want, call))                            # (whose tensors the graph reads)
    for _ in range(3):
        for graph, out, _w, _c in calls:
            for x in out:
                x.zero_()
            graph.replay()
    torch.cuda.synchronize()
    for _g, out, want, _c in calls:
        assert all(torch.equal(x, y) for x, y in zip(out, want))
    assert ws.read_status()[1] == 0


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("Q,strands,depth", [(32, 32, 31), (8, 8, 64), (8, 8, 65), (33, 33, 20), (64, 40, 9), (20, 4, 50)])
def test_strands_of_nodes_that_take_many_rounds(Q, strands, depth, e4m3):
    """Node i hangs on node i - strands: many nodes at each depth, more of them than are looked up at a time, rows that end at any depth."""
    N = strands * depth
    host = ku.Host(2, N + 40, 1, 64, 16, e4m3, seed=Q)
    parent = torch.arange(-strands, N - strands, dtype=I32).clamp(min=-1).repeat(2, 1)
    node = torch.randint(0, N, (2 * Q,), generator=ku.gen(depth)).to(I32)
    node[:Q] = N - 1 - torch.arange(Q, dtype=I32)
    node[Q] = -1
    check(host, ku.bf16((2 * Q, 2, 64), 5), [33, 0], Q, node, parent)


@pytest.mark.parametrize("d,Hq,Hk,Q", [(64, 4, 4, 64), (128, 8, 2, 64), (128, 4, 4, 5), (256, 2, 1, 33)])
def test_a_block_of_tokens_sees_what_lies_in_front(d, Hq, Hk, Q):
    """Row i is node i of a chain: causal attention inside the block."""
    host = ku.Host(3, 300 + Q, Hk, d, 16, False, seed=Q)
    check(host, ku.bf16((3 * Q, Hq, d), 5), [0, 17, 300], Q, torch.arange(Q, dtype=I32).repeat(3))


def test_an_eight_bit_row_that_no_sequence_has_does_not_matter():
    """Not even the cache's first row, marked as no number, where tiles are filled up behind the last token or a page is missing."""
    for Hq, Q in ((2, 1), (16, 1), (64, 1), (2, 3)):
        host = ku.Host(2, 60, 2, 64, 16, True, seed=2)
        free = min(set(range(1, host.k.shape[0])) - set(host.pages.flatten().tolist()))
        for x in (host.k.view(torch.uint8), host.v.view(torch.uint8), host.ke, host.ve):   # page 0's owner, if any, takes a free page
            x[free] = x[0]
        host.pages[host.pages == 0] = free
        host.ke[0], host.ve[0] = 255, 255
        host.k.view(torch.uint8)[0], host.v.view(torch.uint8)[0] = 0x7f, 0xff
        node = None if Q == 1 else torch.tensor([0, 4, -1] * 2, dtype=I32)
        out, _ = check(host, ku.bf16((2 * Q, Hq, 64), 3), [5, 33], Q, node)
        assert bool(torch.isfinite(out).all())
        broken = host.pages.clone()
        broken[1, 1] = -1
        ws = ku.attend_ws(2, Q, Hq, 2, 64)
        out, _ = vt.vt_kv_attend(ku.bf16((2 * Q, Hq, 64), 3).cuda(), host.dev, broken.cuda(), torch.tensor([5, 33], dtype=I32).cuda(),
                                 None if node is None else node.cuda(), ws=ws)
        assert bool(torch.isfinite(out).all()) and ws.read_status()[1] == vt.VT_FLAG_BAD_PAGE
