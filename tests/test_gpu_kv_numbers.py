"""Attention over the paged cache where numbers go to their ends: infinite queries beside missing tokens, powers of values that lie far apart,
light tokens behind heavy ones, bytes that are no number."""
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


@pytest.mark.parametrize("power", [40, 100, -80])
@pytest.mark.parametrize("d,Hq,Q", [(64, 2, 1), (64, 8, 2), (128, 4, 1), (128, 32, 2), (128, 16, 4), (256, 2, 1), (256, 20, 1)])
def test_powers_of_values_that_lie_far_apart(d, Hq, Q, power):
    """Rows of zeros (their power is 2^-126) in front of, behind and between rows of 2^power: a token counts in the sum of weights by its
    score alone.  In one tile, in tiles of several teams and in parts of several CTAs."""
    for n in (32, 64, 65, 300, 3000):
        for order in ("front", "behind", "between", "teams"):
            host = ku.Host(1, n + 8, 1, d, 16, True, seed=n)
            host.ve = torch.full_like(host.ve, 127 + power - 6)
            none = {"front": lambda i: i < n // 2, "behind": lambda i: i >= n // 2, "between": lambda i: i % 2, "teams": lambda i: i // 32 % 2}[order]
            for i in range(n + 8):
                p, j = host.place(0, i)
                if none(i):
                    host.v.view(torch.uint8)[p, :, j], host.ve[p, :, j] = 0, 1
            node = torch.arange(Q, dtype=I32) + 3 if Q > 1 else None
            check(host, ku.bf16((Q, Hq, d), 3), [n], Q, node)


def test_written_rows_of_zeros_count_as_tokens():
    """As a program meets them: rows of zeros and rows of 2^40 through the write, equal scores."""
    cache, pages = vt.kv_cache(5, 1, 16, 64, e4m3=True), torch.arange(4, dtype=I32, device="cuda")[None]
    k = torch.zeros((64, 1, 64), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    v[32:] = 2.0 ** 40
    at = torch.arange(64, dtype=I32, device="cuda")
    q = vt.vt_qkv_write(torch.ones((64, 1, 64), dtype=torch.bfloat16, device="cuda"), k, v, cache, pages, at)
    out, lse = vt.vt_kv_attend(q[:1], cache, pages, at[:1] + 64)
    assert bool((out == 2.0 ** 39).all()) and abs(float(lse) - math.log(64)) < 1e-5


@pytest.mark.parametrize("nats", [8, 15, 16, 17.25, 20])
@pytest.mark.parametrize("d,Hq", [(64, 2), (64, 32), (128, 1), (128, 40), (256, 2)])
def test_light_tokens_behind_heavy_ones(d, Hq, nats):
    """8 tokens e^nats times as heavy as each of the 8184 behind them, one in the first tile of each team, whose values are zero: each of the
    others is tiny beside them, and the result is theirs.  300 sequences of the same pages, so that a CTA's run holds whole results.  Bound: a
    weight is off by 2^-11 of it, or by 2^-36 of the heaviest (times power of its values, the same for all here); scores and
    exponentials by 2^-20; a sum by a step, 2^-23, an addition (fewer than the tokens); out is rounded to bf16."""
    n, S = 8192, 300
    host = ku.Host(1, n, 1, d, 64, True, seed=1)
    host.ke, host.ve = torch.full_like(host.ke, 112), torch.full_like(host.ve, 127 - 7)
    v = host.v.view(torch.uint8)
    v &= 0x7f                                                              # all values at least zero
    scale = nats / (2.0 * d)                                               # queries of one, heavy keys of two
    for i in range(5, 256, 32):
        p, j = host.place(0, i)
        host.k[p, :, j], host.ke[p, :, j] = torch.tensor(2.0).to(torch.float8_e4m3fn), 127
        host.v.view(torch.uint8)[p, :, j] = 0
    dev = host.device()
    out, lse = vt.vt_kv_attend(torch.ones((S, Hq, d), dtype=torch.bfloat16, device="cuda"), dev, host.pages_dev.expand(S, -1).contiguous(),
                               torch.full((S,), n, dtype=I32, device="cuda"), scale=scale)
    k, vv = host.values(0, list(range(n)))
    z = k[:, 0].sum(1) * scale
    w = torch.softmax(z, 0)
    ref = (w[:, None] * vv[:, 0]).sum(0)
    steps = n * 2.0 ** -23
    tol = (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -20 + 2 * steps + 2.0 ** -19) * ref + n * 2.0 ** -36 * 448 * 2.0 ** -7 * float(w.max())
    off = (out.double().cpu() - ref).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
    assert float((lse.double().cpu() - torch.logsumexp(z, 0)).abs().max()) <= 2.0 ** -19 + steps + 2.0 ** -22 * 30


def test_bytes_that_are_no_number():
    """0x7f and 0xff, which the write never makes, read as NaN wherever they lie: in a committed token, and in a drafted one for the rows
    that see it, a key's for all dims, a value's for its own."""
    for Hq, Q, d in ((4, 4, 64), (32, 5, 128), (8, 5, 256), (1, 4, 128)):
        for what in ("k", "v"):
            for byte in (0x7f, 0xff):
                for place in (3, 21 + 0):                                  # committed; node 0, which rows of nodes 4 and 2 see
                    host = ku.Host(1, 60, 1, d, 16, True, seed=11)
                    parent = torch.tensor([[-1, -1, 0, 1, 2, 3]], dtype=I32)
                    node = torch.tensor([4, 5, 2, 3, -1][:Q], dtype=I32)
                    q = ku.bf16((Q, Hq, d), 3)
                    p, j = host.place(0, place)
                    x = host.k if what == "k" else host.v
                    x.view(torch.uint8)[p, 0, j, 37] = 0
                    ref, ref_l, tol, tol_l = ku.attend(host, q, [21], Q, node, parent)
                    sees = torch.ones(Q, dtype=torch.bool) if place == 3 else torch.tensor([True, False, True, False, False][:Q])
                    if what == "k":
                        ref[sees], ref_l[sees] = math.nan, math.nan
                    else:
                        ref[sees, :, 37] = math.nan
                    x.view(torch.uint8)[p, 0, j, 37] = byte
                    out, lse = vt.vt_kv_attend(q.cuda(), host.device(), host.pages_dev, torch.tensor([21], dtype=I32).cuda(), node.cuda(), parent.cuda())
                    assert ku.near(out, ref, tol)[0] and ku.near(lse, ref_l, tol_l)[0], (Hq, Q, d, what, byte, place)
                    k, v = vt.vt_kv_read(host.dev, host.pages_dev, torch.tensor([place], dtype=I32).cuda())
                    assert bool(torch.isnan((k if what == "k" else v)[0, 0, 37]))
