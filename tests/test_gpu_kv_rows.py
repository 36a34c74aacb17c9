"""Rows of the paged cache: written (norms, rotation, 8-bit rows), read back and moved, against the same steps in 64 bits.

Bytes of an 8-bit cache are compared for equality: they are roundings of values computed in 64 bits, and no value of these inputs lies within
their error of a border."""
import math

import numpy as np
import pytest
import torch

import kv_util as ku
import paper_2506_22694_b200 as vt

pytestmark = pytest.mark.gpu
I32 = torch.int32


def write(host, T, Hq, index, seq, positions, rot=0, interleaved=False, norm=False, base=10000.0, eps=1e-6, seed=1, std=1.0, wide=True, ws=None, flags=0, data=None):
    d, Hk = host.d, host.heads
    if data is None:
        x = ku.bf16((T, (Hq + 2 * Hk) * d), seed, std)
    else:
        x = data
    q, k, v = (y.view(T, -1, d) for y in x.split([Hq * d, Hk * d, Hk * d], 1))
    xd = x.cuda()
    qd, kd, vd = (y.view(T, -1, d) for y in xd.split([Hq * d, Hk * d, Hk * d], 1))
    if not wide:
        qd, kd, vd = qd.contiguous(), kd.contiguous(), vd.contiguous()
    qw, kw = ((1 + ku.bf16((d,), s, 0.2).float()).to(torch.bfloat16) for s in (91, 92)) if norm else (None, None)
    freqs = vt.vt_rope_freqs(rot, base) if rot else None
    dev = host.device()
    index, positions = torch.tensor(index, dtype=I32), torch.tensor(positions, dtype=I32)
    ws = ws or vt.Workspace(vt.VT_CTRL_BYTES)
    got = vt.vt_qkv_write(qd if Hq else None, kd, vd, dev, host.pages_dev, index.cuda(), None if seq is None else torch.tensor(seq, dtype=I32).cuda(),
                          positions.cuda(), freqs, q_weight=None if qw is None else qw.cuda(), k_weight=None if kw is None else kw.cuda(), eps=eps,
                          interleaved=interleaved, ws=ws)
    seq = [t // (T // host.S) for t in range(T)] if seq is None else seq
    yq, tol, yk, ktol = ku.written(host, q if Hq else None, k, v, index, seq, positions, ku.inv_freq(rot, base) if rot else None, interleaved, qw, kw, eps)
    if Hq:
        ok, worst = ku.near(got, yq, tol)
        assert ok, "q is %.3g of its bound off" % worst
    else:
        assert got is None
    if not host.e4m3:                                                    # the written keys against their bound, then as they are
        there = dev[0].cpu()
        for t in range(T):
            s, i = int(seq[t]), int(index[t])
            if 0 <= i < host.pages.shape[1] * host.page and 0 <= s < host.S:
                p, j = host.place(s, i)
                if 0 <= p < there.shape[0]:
                    ok, worst = ku.near(there[p, :, j], yk[t], ktol[t])
                    assert ok, "k is %.3g of its bound off" % worst
                    host.k[p, :, j] = there[p, :, j]
    assert host.same()
    assert ws.read_status()[1] == flags
    return got


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d,Hq,Hk,page,rot,interleaved,norm", [
    (64, 8, 8, 16, 64, False, False), (64, 32, 8, 7, 32, False, True), (96, 12, 12, 16, 96, False, True), (96, 4, 4, 8, 48, True, False),
    (128, 8, 8, 16, 128, False, False), (128, 32, 8, 64, 128, False, True), (128, 28, 4, 5, 64, True, True), (128, 7, 1, 16, 0, False, True),
    (192, 6, 2, 24, 192, False, True), (256, 16, 2, 16, 256, False, True), (256, 3, 3, 1, 16, True, False), (128, 0, 5, 16, 128, False, True)])
def test_write(d, Hq, Hk, page, rot, interleaved, norm, e4m3):
    host = ku.Host(3, 40, Hk, d, page, e4m3, seed=d, layout="nphd" if page == 16 else "nhpd")
    seq = [2, 0, 0, 1, 2, 2, 1]
    index = [0, 5, 6, 39, 17, 16, -1]
    positions = [0, 1, 77, 4095, 131071, -3, 2 ** 31 - 1]                  # (far ones: nothing is lost)
    write(host, 7, Hq, index, seq, positions, rot, interleaved, norm, wide=d != 64)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("S,rows,Hq,Hk,d", [(1, 1, 8, 8, 128), (5, 1, 32, 8, 128), (3, 8, 8, 2, 64), (2, 61, 4, 4, 128)])
def test_write_rows_of_each_sequence_in_order(S, rows, Hq, Hk, d, e4m3):
    host = ku.Host(S, 20 + rows, Hk, d, 16, e4m3, seed=3)
    write(host, S * rows, Hq, [20 - s % 3 + r for s in range(S) for r in range(rows)], None, [7 + r for _ in range(S) for r in range(rows)], d, norm=True, wide=False)


def test_write_a_prompt_of_many_tokens():
    """More tokens than the chip has seats for."""
    for e4m3 in (False, True):
        host = ku.Host(1, 2600, 1, 64, 64, e4m3, seed=3)
        write(host, 2600, 9, list(range(2600)), None, list(range(2600)), 64, norm=True, base=500000.0)


def test_eight_bit_rows_at_their_edges():
    """Ties between two values, largest magnitudes at and next to 448 times a power of two, subnormal, zero and huge rows, NaN and infinities."""
    d = 64
    rows = []
    grid = torch.tensor(ku.E4M3[:127], dtype=torch.float64)
    ties = ((grid[1:] + grid[:-1]) / 2).float()
    for e in (-100, -9, 0, 5, 100):
        x = torch.zeros(d)
        x[0] = 448.0 * 2.0 ** e
        x[1:] = ties[torch.arange(63) * 2] * 2.0 ** e * torch.where(torch.arange(63) % 2 == 0, 1.0, -1.0)
        rows.append(x)
        y = x.clone()
        y[0] = 450.0 * 2.0 ** e                                           # the next bf16 above
        rows.append(y)
        y = x.clone()
        y[0], y[1] = 446.0 * 2.0 ** e, 0.0
        rows.append(y)
    rows.append(torch.zeros(d))
    rows.append(-torch.zeros(d))
    rows.append(torch.full((d,), 2.0 ** -133))                            # bf16 subnormals: below the smallest power
    rows.append(torch.linspace(-3.3e38, 3.3e38, d))
    for bad in (math.nan, math.inf, -math.inf):
        x = torch.linspace(-1, 1, d)
        x[17] = bad
        rows.append(x)
    v = torch.stack(rows).to(torch.bfloat16)
    T = v.shape[0]
    data = torch.cat([v, v.flip(0)], 1)
    host = ku.Host(1, T, 1, d, 16, True, seed=4)
    write(host, T, 0, list(range(T)), None, [0] * T, data=data)
    k, vv = vt.vt_kv_read(host.dev, host.pages_dev, torch.arange(T, dtype=I32).cuda())
    ref = torch.stack([host.values(0, [t])[1][0] for t in range(T)])
    assert torch.equal(torch.isnan(vv.cpu()), torch.isnan(ref))
    fine = ~torch.isnan(ref)
    assert torch.equal(vv.cpu().double()[fine], ref[fine])                # (a row read back is exact in bf16)


def test_the_sum_of_a_wide_row_and_eps():
    """Rows of tiny, huge and equal entries through the norm."""
    for e4m3 in (False, True):
        host = ku.Host(1, 8, 2, 256, 8, e4m3, seed=6)
        x = ku.bf16((6, (2 + 4) * 256), 3)
        x[1] *= 2.0 ** -60
        x[2] *= 2.0 ** 50
        x[3] = 0
        x[4] = 1.0
        write(host, 6, 2, list(range(6)), None, [3] * 6, 256, norm=True, eps=1e-5, data=x)


def test_infinities_stay_in_their_pair_and_out_of_the_unrotated_dims():
    host = ku.Host(1, 8, 1, 128, 8, False, seed=6)
    x = ku.bf16((2, 3 * 128), 3)
    x[0, 3] = math.inf                                                    # of q: its partner is dim 35
    freqs = vt.vt_rope_freqs(64)
    dev = host.device()
    q, k, v = (y.view(2, 1, 128) for y in x.cuda().split(128, 1))
    got = vt.vt_qkv_write(q, k, v, dev, host.pages_dev, torch.tensor([0, 1], dtype=I32).cuda(), None, torch.tensor([5, 6], dtype=I32).cuda(), freqs)
    bad = (~torch.isfinite(got.float())).nonzero().tolist()
    assert bad == [[0, 0, 3], [0, 0, 35]]


def test_write_leaves_out_what_is_out_of_range_and_says_so():
    for e4m3 in (False, True):
        host = ku.Host(2, 30, 2, 64, 10, e4m3, seed=9)
        host.pages[1, 2] = host.k.shape[0]
        ws = vt.Workspace(vt.VT_CTRL_BYTES)
        write(host, 3, 4, [1, -1, -2 ** 31], [0, 0, 5], [0, 0, 0], 64, ws=ws)                  # (negative places are nobody's error)
        for seq, index in ((2, 0), (-1, 0), (0, 30), (0, 2 ** 31 - 1), (1, 25)):
            write(host, 2, 4, [index, 3], [seq, 1], [1, 2], 64, ws=ws, flags=vt.VT_FLAG_BAD_PAGE)
        for page in (-1, -2, -2 ** 31):
            host.pages[1, 2] = page
            write(host, 2, 4, [25, 3], [1, 1], [1, 2], 64, ws=ws, flags=vt.VT_FLAG_BAD_PAGE)


def test_queries_in_place():
    host = ku.Host(1, 8, 2, 128, 8, False, seed=6)
    x = ku.bf16((5, 8 * 128), 3).view(5, 8, 128).cuda()
    k = ku.bf16((5, 2 * 128), 4).view(5, 2, 128).cuda()
    dev, at, freqs = host.device(), torch.arange(5, dtype=I32).cuda(), vt.vt_rope_freqs(128)
    ref = vt.vt_qkv_write(x, k, k, dev, host.pages_dev, at, None, at, freqs)
    got = vt.vt_qkv_write(x, k, k, dev, host.pages_dev, at, None, at, freqs, out=x)
    assert got is x and torch.equal(got, ref)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d,Hk,page", [(64, 8, 16), (96, 3, 7), (128, 8, 64), (192, 2, 1), (256, 5, 16), (128, 1, 16)])
def test_read(d, Hk, page, e4m3):
    host = ku.Host(3, 50, Hk, d, page, e4m3, seed=d + 1, layout="nphd" if page == 7 else "nhpd")
    dev = host.device()
    seq = [0, 1, 2, 2, 1, 0, 0, 3, -1, 1]
    index = [49, 0, 17, 18, -1, 16, 2 ** 31 - 1, 0, 0, 33]
    ws = vt.Workspace(vt.VT_CTRL_BYTES)
    k, v = vt.vt_kv_read(dev, host.pages_dev, torch.tensor(index, dtype=I32).cuda(), torch.tensor(seq, dtype=I32).cuda(), ws=ws)
    for t, (s, i) in enumerate(zip(seq, index)):
        if 0 <= s < 3 and 0 <= i < 50:
            rk, rv = host.values(s, [i])
            assert torch.equal(k[t].cpu().double(), rk[0]) and torch.equal(v[t].cpu().double(), rv[0])
        else:
            assert not k[t].any() and not v[t].any()
    assert ws.read_status()[1] == vt.VT_FLAG_BAD_PAGE
    k, v = vt.vt_kv_read(dev, host.pages_dev, torch.arange(6, dtype=I32).cuda() % 2)              # two rows of each in order
    for t in range(6):
        rk, rv = host.values(t // 2, [t % 2])
        assert torch.equal(k[t].cpu().double(), rk[0]) and torch.equal(v[t].cpu().double(), rv[0])
    empty = vt.vt_kv_read(dev, host.pages_dev, torch.empty(0, dtype=I32).cuda())
    assert empty[0].shape == (0, Hk, d)


def move(host, lens, path, n_accept, nodes=None):
    """The moves one after the other."""
    for s in range(host.S):
        n = int(n_accept[s])
        if int(lens[s]) < 0 or n < 0 or n > path.shape[1]:
            continue
        for i in range(n):
            f = int(path[s, i])
            f = int(nodes[s, f]) if nodes is not None else f
            a, b = host.place(s, int(lens[s]) + f), host.place(s, int(lens[s]) + i)
            for x in (host.k, host.v, host.ke, host.ve):
                if x is not None:
                    x = x.view(torch.uint8) if host.e4m3 else x
                    x[b[0], :, b[1]] = x[a[0], :, a[1]].clone()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("S,N,d,Hk,page", [(1, 7, 128, 8, 16), (4, 60, 64, 2, 16), (3, 32, 128, 8, 5), (2, 300, 256, 1, 16), (40, 9, 96, 3, 8)])
def test_commit(S, N, d, Hk, page, e4m3):
    host = ku.Host(S, 40 + 2 * N, Hk, d, page, e4m3, seed=N, layout="nphd" if page == 5 else "nhpd")
    g = ku.gen(S + N)
    lens = torch.randint(0, 40, (S,), generator=g).to(I32)
    n_accept = torch.randint(0, N + 1, (S,), generator=g).to(I32)
    path = torch.full((S, N), -1, dtype=I32)
    nodes = torch.sort(torch.rand((S, 2 * N), generator=g).argsort(1)[:, :N], 1)[0].to(I32)
    for s in range(S):
        n = int(n_accept[s])
        path[s, :n] = torch.sort(torch.randperm(N, generator=g)[:n])[0].to(I32)
    for use in (None, nodes):
        dev = host.device()
        ws = vt.Workspace(vt.VT_CTRL_BYTES)
        got = vt.vt_kv_commit(dev, host.pages_dev, lens.cuda(), path.cuda(), n_accept.cuda(), None if use is None else use.cuda(), ws=ws)
        move(host, lens, path, n_accept, use)
        assert host.same() and ws.read_status()[1] == 0
        assert torch.equal(got.cpu(), lens + n_accept)


def test_commit_in_place_of_the_lengths_and_of_what_is_out_of_range():
    host = ku.Host(5, 40, 2, 64, 16, False, seed=2)
    lens = torch.tensor([3, 5, -1, 2, 38], dtype=I32)
    n_accept = torch.tensor([2, 9, 1, -3, 1], dtype=I32)
    path = torch.tensor([[4, 1, -1, -1, -1]] * 5, dtype=I32)               # path[1] = 1 stays where it is
    host.pages[4, 2] = -1                                                  # (place 42 of the last sequence: beyond its pages)
    dev = host.device()
    ws = vt.Workspace(vt.VT_CTRL_BYTES)
    ld = lens.cuda()
    got = vt.vt_kv_commit(dev, host.pages_dev, ld, path.cuda(), n_accept.cuda(), out=ld, ws=ws)
    move(host, lens[:1].tolist() + [0] * 4, path, [2, 0, 0, 0, 0])
    assert got is ld and got.cpu().tolist() == [5, 5, -1, 2, 39]
    assert host.same() and ws.read_status()[1] == vt.VT_FLAG_BAD_PAGE
    bad = torch.tensor([[4, 0, 9, -1]] * 5, dtype=I32)                     # node 0 in place 1, node 9 of 4: left out
    vt.vt_kv_commit(dev, host.pages_dev, torch.tensor([3, 0, 0, 0, 0], dtype=I32).cuda(), bad.cuda(), torch.tensor([3, 0, 0, 0, 0], dtype=I32).cuda(), ws=ws)
    move(host, [3, 0, 0, 0, 0], bad, [1, 0, 0, 0, 0])
    assert host.same() and ws.read_status()[1] == vt.VT_FLAG_BAD_PAGE


def test_frequencies_of_a_stretched_context():
    """Llama 3's rule: short wavelengths as they are, long ones by the factor, in between in proportion."""
    rot, base, factor, lo, hi, original = 128, 500000.0, 8.0, 1.0, 4.0, 8192.0
    got = vt.vt_rope_freqs(rot, base, factor, lo, hi, original, device="cpu")
    f = ku.inv_freq(rot, base).numpy()
    wave = 2 * np.pi / f
    keep = np.clip((original / wave - lo) / (hi - lo), 0, 1)
    want = (1 - keep) * f / factor + keep * f
    assert np.allclose(got.numpy() / 2.0 ** 64 * 2 * np.pi, want, rtol=1e-13, atol=1e-18)
    assert np.allclose(vt.vt_rope_freqs(rot, base, device="cpu").numpy() / 2.0 ** 64 * 2 * np.pi, f, rtol=1e-13, atol=1e-18)


def test_no_tokens_and_no_sequences():
    for e4m3 in (False, True):
        host = ku.Host(2, 20, 2, 64, 16, e4m3, seed=2)
        dev = host.device()
        none = torch.empty(0, dtype=I32, device="cuda")
        q, k = (torch.empty((0, h, 64), dtype=torch.bfloat16, device="cuda") for h in (4, 2))
        for pages in (host.pages_dev, host.pages_dev[:0]):
            assert vt.vt_qkv_write(q, k, k, dev, pages, none, None, none, vt.vt_rope_freqs(64)).shape == (0, 4, 64)
            assert vt.vt_kv_read(dev, pages, none)[1].shape == (0, 2, 64)
        path = torch.empty((0, 5), dtype=I32, device="cuda")
        assert vt.vt_kv_commit(dev, host.pages_dev[:0], none, path, none).shape == (0,)
        assert host.same()
