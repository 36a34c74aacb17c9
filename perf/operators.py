"""The drafter's attention over its paged key-value cache, as cases that can be timed and compared.

A drafting loop runs, between two calls of the trimmed head, the attention of the rows that it drafts: queries and keys get their
per-head norm and rotation and keys and values go into the cache (kind "write"), the rows attend to the committed tokens and to
their ancestors in the draft tree ("attend"), and once the target has verified a block the accepted path becomes part of the
committed tokens ("commit").  A program that reuses a prefix elsewhere reads cached rows back ("read").

Caches hold bf16, or e4m3 with one power of two per token and head.  Head layouts are those of the drafters that the benchmark
names (8 heads of 128 over a hidden size of 1024; 32 query and 8 key heads of 128 over 4096, of 64 over 2048) and others of the
same kind; trees are the paper's (top-8 and top-10, depths 3 to 6).
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
EPS = 1e-6
BASE = 500000.0


# ---- cases -------------------------------------------------------------------------------------------
def _write(name, S, rows, length, Hq, Hk, D, page, e4m3, norm, rot):
    """`rows` new tokens of each of S sequences behind `length` cached ones (0 rows: a prompt of `length` tokens each)."""
    return {"name": name, "kind": "write", "S": S, "rows": rows, "length": length, "Hq": Hq, "Hk": Hk, "D": D, "page": page,
            "e4m3": e4m3, "norm": norm, "rot": rot}


def _read(name, S, length, Hk, D, page, e4m3):
    return {"name": name, "kind": "read", "S": S, "length": length, "Hk": Hk, "D": D, "page": page, "e4m3": e4m3}


def _attend(name, S, Q, nodes, length, Hq, Hk, D, page, e4m3):
    """Q rows a sequence; nodes: size of a sequence's draft tree (0: rows see the committed tokens alone)."""
    return {"name": name, "kind": "attend", "S": S, "Q": Q, "nodes": nodes, "length": length, "Hq": Hq, "Hk": Hk, "D": D, "page": page,
            "e4m3": e4m3}


def _commit(name, S, nodes, length, Hk, D, page, e4m3):
    return {"name": name, "kind": "commit", "S": S, "nodes": nodes, "length": length, "Hk": Hk, "D": D, "page": page, "e4m3": e4m3}


def listed():
    return [
        # one draft token of one sequence of the small drafter: latency
        _write("write_token", 1, 1, 700, 8, 8, 128, 16, False, False, 128),
        # a depth of four nodes for 64 sequences, query and key norms, cache in 8 bits
        _write("write_frontier_e4m3", 64, 4, 1000, 32, 8, 128, 32, True, True, 128),
        # prompts of seven users, all tokens at once
        _write("write_prompt", 7, 0, 2041, 32, 8, 128, 64, False, True, 128),
        # a short shared prefix handed to another program
        _read("read_prefix", 3, 911, 8, 128, 16, False),
        # the caches of a batch, taken back from 8 bits
        _read("read_batch_e4m3", 29, 6007, 8, 128, 64, True),
        # one draft token over a short conversation: latency
        _attend("attend_token", 1, 1, 0, 701, 8, 8, 128, 16, False),
        # one depth of a tree: ten nodes with their ancestors behind 4001 committed tokens
        _attend("attend_tree", 1, 10, 310, 4001, 32, 8, 128, 16, False),
        # one draft token over a very long document, cache in 8 bits
        _attend("attend_long_e4m3", 1, 1, 0, 131_071, 32, 8, 128, 64, True),
        # a draft token of each of 64 conversations of very different lengths
        _attend("attend_batch", 64, 1, 0, 8000, 32, 8, 128, 32, False),
        # a tree depth of eight nodes for 32 conversations, heads of 64, cache in 8 bits
        _attend("attend_batch_tree_e4m3", 32, 8, 136, 6000, 32, 8, 64, 32, True),
        # the accepted path of one verified tree
        _commit("commit_block", 1, 60, 2000, 8, 128, 16, False),
        # accepted paths of a batch, cache in 8 bits
        _commit("commit_batch_e4m3", 256, 32, 500, 8, 128, 32, True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    kind = rng.choice(["write", "write", "read", "attend", "attend", "attend", "attend", "commit"])
    Hq, Hk, D = rng.choice([(8, 8, 128), (32, 8, 128), (32, 8, 64), (28, 4, 128), (16, 2, 256), (24, 8, 128), (12, 12, 96)])
    page, e4m3 = rng.choice([16, 16, 32, 64, 64, 128, 24, 8]), rng.random() < 0.5
    if kind == "write":
        norm, rot = rng.random() < 0.5, rng.choice([D, D, D // 2])
        if rng.random() < 0.3:
            S = _log(rng, 1, 16)
            c = _write("", S, 0, _log(rng, 17, 16_000 // S), Hq, Hk, D, page, e4m3, norm, rot)
        else:
            c = _write("", _log(rng, 1, 128), rng.choice([1, 1, 4, 8, 10]), _log(rng, 1, 4000), Hq, Hk, D, page, e4m3, norm, rot)
    elif kind == "read":
        S = _log(rng, 1, 64)
        c = _read("", S, _log(rng, 1, 120_000 // S), Hk, D, page, e4m3)
    elif kind == "attend":
        S = _log(rng, 1, 96)
        Q = rng.choice([1, 1, 1, 4, 8, 10, 16, 60])
        nodes = 0 if Q == 1 and rng.random() < 0.7 else rng.randint(Q, 4 * Q + 60)
        c = _attend("", S, Q, nodes, _log(rng, 1, 200_000 // S if Q < 60 else 40_000 // S), Hq, Hk, D, page, e4m3)
    else:
        c = _commit("", _log(rng, 1, 256), rng.choice([7, 32, 60, rng.randint(2, 90)]), _log(rng, 1, 1000), Hk, D, page, e4m3)
    del c["name"]
    return c


def _lengths(case):
    """Committed tokens of each sequence: ragged, from a sixteenth of the longest up; every ninth slot of a batch is idle."""
    S, top = case["S"], case["length"]
    out = []
    for s in range(S):
        part = 1.0 if s == 0 else 0.0625 + 0.9375 * ((s * 0.6180339887498949) % 1.0)
        out.append(0 if s % 9 == 8 else max(1, round(top * part)))
    return out


# ---- inputs ------------------------------------------------------------------------------------------
def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * int(seed) + salt)
    return g


def _gauss(shape, std, g):
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(0.0, std, generator=g)


def _two_to(e):
    """2^e for whole e in [-126, 127], by its bits (a power function need not be exact)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _exponent(amax):
    """Smallest e with amax <= 448 * 2^e, at least -126 (amax = m * 2^x with m in [0.5, 1), and 448 = 0.875 * 2^9)."""
    m, x = torch.frexp(amax)
    return torch.where(amax > 0, torch.where(m <= 0.875, x - 9, x - 8), torch.full_like(x, -126)).clamp(min=-126)


def _round_e4m3(x):
    """x (64 bits, at most 448) to the nearest value of four exponent and three mantissa bits, ties to even."""
    step = _two_to((torch.frexp(x.abs())[1] - 1).clamp(min=-6) - 3).double()
    return torch.round(x / step) * step


def _quantise(x):
    """[..., D] -> (e4m3 values, biased exponents) of its rows."""
    x = x.double()
    e = _exponent(x.abs().amax(-1))
    return _round_e4m3(x * _two_to(-e)[..., None].double()).float().to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _cache(case, g):
    """A cache whose pages lie in any order, full of what earlier tokens left: (k, v, k_exp, v_exp) and the page table."""
    S, Hk, D, page = case["S"], case["Hk"], case["D"], case["page"]
    room = case["length"] + case.get("nodes", 0) + case.get("rows", 0) + 1
    per = -(-room // page)
    n = S * per + 3
    pages = torch.randperm(n, generator=g, device=DEV)[: S * per].view(S, per).to(torch.int32)
    k, v = _gauss((n, Hk, page, D), 1.0, g), _gauss((n, Hk, page, D), 0.5, g)
    k[..., ::16] *= 3.0                                    # keys have a few large channels
    if not case["e4m3"]:
        return (k, v, None, None), pages
    (k, ke), (v, ve) = _quantise_large(k), _quantise_large(v)
    return (k, v, ke, ve), pages


def _quantise_large(x):
    q, e = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(x.shape[:-1], dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 25) // max(1, x[0].numel()))
    for i in range(0, x.shape[0], step):
        q[i:i + step], e[i:i + step] = _quantise(x[i:i + step])
    return q, e


def _trees(S, N, Q, g):
    """Parents of N nodes as a tree is expanded (a first depth of W nodes, then W children of each of W nodes a depth), and Q nodes
    of each tree that are drafted from, in pool order."""
    W = 10 if Q == 10 else 8
    i = torch.arange(N, device=DEV)
    depth = torch.where(i < W, 0, 1 + (i - W) // (W * W))
    first = torch.where(depth > 1, W + (depth - 2) * W * W, 0)                  # first node of the depth before, and how many it has
    count = torch.where(depth > 1, W * W, W)
    pick = first + (torch.rand((S, N), generator=g, device=DEV) * count).long().clamp(max=W * W - 1)
    parent = torch.where(depth > 0, pick, -1)
    node = torch.sort(torch.argsort(torch.rand((S, N), generator=g, device=DEV), 1)[:, :Q], 1)[0]
    return parent.to(torch.int32).contiguous(), node.reshape(-1).to(torch.int32)


def prepare(case, seed):
    g = _gen(seed, 3)
    S, Hk, D, kind = case["S"], case["Hk"], case["D"], case["kind"]
    cache, pages = _cache(case, g)
    lens = _lengths(case)
    st = {"case": case, "cache": cache, "pages": pages, "lens": torch.tensor(lens, dtype=torch.int32, device=DEV)}
    if kind == "write":
        if case["rows"]:
            per, first = [case["rows"]] * S, lens
        else:
            per, first = lens, [0] * S
        T, Hq = sum(per), case["Hq"]
        n = torch.tensor(per, device=DEV)
        seq = torch.repeat_interleave(torch.arange(S, device=DEV), n)
        row = torch.arange(T, device=DEV) - torch.repeat_interleave(torch.cumsum(n, 0) - n, n)
        index = torch.tensor(first, device=DEV)[seq] + row
        qkv = _gauss((T, (Hq + 2 * Hk) * D), 1.5, g)        # the projection's output: its heads side by side
        st["q"], st["k"], st["v"] = (x.view(T, -1, D) for x in qkv.split([Hq * D, Hk * D, Hk * D], 1))
        st["seq"], st["index"] = seq.to(torch.int32), index.to(torch.int32)
        st["positions"] = (index + (100_000 if S == 1 else 0)).to(torch.int32)  # (a window far into a document)
        st["qw"], st["kw"] = (1.0 + _gauss((D,), 0.1, g), 1.0 + _gauss((D,), 0.1, g)) if case["norm"] else (None, None)
        st["inv_freq"] = BASE ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=DEV) / case["rot"])
    elif kind == "read":
        n = torch.tensor(lens, device=DEV)
        seq = torch.repeat_interleave(torch.arange(S, device=DEV), n)
        st["seq"] = seq.to(torch.int32)
        st["index"] = (torch.arange(int(n.sum()), device=DEV) - torch.repeat_interleave(torch.cumsum(n, 0) - n, n)).to(torch.int32)
    elif kind == "attend":
        st["q"] = _gauss((S * case["Q"], case["Hq"], D), 1.3, g)
        st["node"] = st["parent"] = None
        if case["nodes"]:
            st["parent"], st["node"] = _trees(S, case["nodes"], case["Q"], g)
    else:
        N = case["nodes"]
        coin = torch.rand((S, N), generator=g, device=DEV)
        st["n_accept"] = (1 + torch.floor(7 * torch.rand(S, generator=g, device=DEV))).clamp(max=N).to(torch.int32)
        order = torch.sort(torch.argsort(coin, 1)[:, :8].to(torch.int32), 1)[0]  # a rising path
        path = torch.full((S, N), -1, dtype=torch.int32, device=DEV)
        path[:, : order.shape[1]] = order
        st["path"] = torch.where(torch.arange(N, device=DEV)[None] < st["n_accept"][:, None], path, torch.full_like(path, -1))
    if own:
        import paper_2506_22694_b200 as vt

        if kind == "write":
            st["freqs"] = vt.vt_rope_freqs(case["rot"], BASE, device=DEV)
        if kind == "attend":
            st["ws"] = vt.Workspace(vt.workspace_bytes(vt.VT_OP_KV_ATTEND, n=S, B=case["Q"], K=case["Hq"], V=Hk, d=D), DEV)
    return st


# ---- the plain forms -----------------------------------------------------------------------------------
def _slots(pages, seq, index, page):
    """Pages, and places in them, of tokens `index` of sequences `seq`."""
    index, seq = index.long(), seq.long()
    return pages[seq, index // page].long(), index % page


def _values(stored, exps, where):
    """Cached rows of all heads at (page, place), in 32 bits: [..., heads, D]."""
    if exps is None:
        return stored[where[0], :, where[1]].float()
    x = stored.view(torch.uint8)[where[0], :, where[1]].view(torch.float8_e4m3fn).float()
    return x * _two_to(exps[where[0], :, where[1]].int() - 127)[..., None]


def _normed(x, w):
    return x if w is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.to(x.dtype)


def _rotated(x, cos, sin):
    half = cos.shape[-1]
    a, b = x[..., :half], x[..., half: 2 * half]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]], -1)


def _plain_write(s):
    angle = (s["positions"].double()[:, None] * s["inv_freq"])[:, None]         # (far positions: in 64 bits)
    cos, sin = torch.cos(angle), torch.sin(angle)
    q = _rotated(_normed(s["q"].float(), s["qw"]), cos.float(), sin.float()).bfloat16()
    at = _slots(s["pages"], s["seq"], s["index"], s["case"]["page"])
    ck, cv, ek, ev = s["cache"]
    if not s["case"]["e4m3"]:
        ck[at[0], :, at[1]] = _rotated(_normed(s["k"].float(), s["kw"]), cos.float(), sin.float()).bfloat16()
        cv[at[0], :, at[1]] = s["v"]
        return q, ck, cv
    k, ek[at[0], :, at[1]] = _quantise(_rotated(_normed(s["k"].double(), s["kw"]), cos, sin))   # (next to a border: in 64 bits)
    v, ev[at[0], :, at[1]] = _quantise(s["v"])
    ck.view(torch.uint8)[at[0], :, at[1]] = k.view(torch.uint8)
    cv.view(torch.uint8)[at[0], :, at[1]] = v.view(torch.uint8)
    return q, _values(ck, ek, at).bfloat16(), _values(cv, ev, at).bfloat16()


def _plain_read(s):
    ck, cv, ek, ev = s["cache"]
    at = _slots(s["pages"], s["seq"], s["index"], s["case"]["page"])
    return _values(ck, ek, at).bfloat16(), _values(cv, ev, at).bfloat16()


def _plain_attend(s):
    case, lens = s["case"], s["lens"].long()
    S, Q, Hk, D, N = case["S"], case["Q"], case["Hk"], case["D"], case["nodes"]
    top = case["length"]
    column = torch.arange(top + N, device=DEV)[None].expand(S, -1)              # the committed tokens, then the nodes
    index = torch.where(column < top, column, lens[:, None] + column - top)
    sees = (column < torch.minimum(lens, torch.full_like(lens, top))[:, None])[:, None].repeat(1, Q, 1)
    if N:
        edge = (s["parent"].long()[:, :, None] == torch.arange(N, device=DEV)).float()
        above = torch.linalg.matrix_power(edge + torch.eye(N, device=DEV), 16) > 0   # [S, node, its ancestors and itself]
        sees[:, :, top:] = above[torch.arange(S, device=DEV)[:, None], s["node"].view(S, Q).long()]
    at = _slots(s["pages"], torch.arange(S, device=DEV)[:, None], index, case["page"])
    ck, cv, ek, ev = s["cache"]
    k = _values(ck, ek, at)
    q = s["q"].float().view(S, Q, Hk, -1, D)
    score = torch.einsum("sqhgd,sphd->shgqp", q, k) / math.sqrt(D)
    del k
    score = score.masked_fill(~sees[:, None, None], -math.inf)
    most = score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(score - most)
    total = p.sum(-1)
    out = torch.einsum("shgqp,sphd->sqhgd", p, _values(cv, ev, at))
    some = total.permute(0, 3, 1, 2)[..., None]
    out = torch.where(some > 0, out / some.clamp(min=1e-37), torch.zeros_like(out))
    lse = (torch.log(total) + most[..., 0]).permute(0, 3, 1, 2)
    return out.reshape(S * Q, -1, D).bfloat16(), torch.where(some[..., 0] > 0, lse, torch.full_like(lse, -math.inf)).reshape(S * Q, -1)


def _plain_commit(s):
    case, N = s["case"], s["case"]["nodes"]
    i = torch.arange(N, device=DEV)[None]
    seq, i = torch.nonzero(i < s["n_accept"][:, None], as_tuple=True)
    src = _slots(s["pages"], seq, s["lens"][seq] + s["path"][seq, i], case["page"])
    dst = _slots(s["pages"], seq, s["lens"][seq] + i, case["page"])
    for x in s["cache"]:
        if x is not None:
            x = x.view(torch.uint8) if case["e4m3"] else x
            x[dst[0], :, dst[1]] = x[src[0], :, src[1]]
    return [x for x in s["cache"] if x is not None], s["lens"] + s["n_accept"]


PLAIN = {"write": _plain_write, "read": _plain_read, "attend": _plain_attend, "commit": _plain_commit}


# ---- one pass ------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return PLAIN[kind](s)
    import paper_2506_22694_b200 as vt

    if kind == "write":
        seq = None if case["rows"] else s["seq"]                                # (equal numbers of rows lie in the sequences' order)
        q = vt.vt_qkv_write(s["q"], s["k"], s["v"], s["cache"], s["pages"], s["index"], seq, s["positions"], s["freqs"],
                            q_weight=s["qw"], k_weight=s["kw"], eps=EPS)
        if case["e4m3"]:
            return q, *vt.vt_kv_read(s["cache"], s["pages"], s["index"], seq)
        return q, s["cache"][0], s["cache"][1]
    if kind == "read":
        return vt.vt_kv_read(s["cache"], s["pages"], s["index"], s["seq"])
    if kind == "attend":
        return vt.vt_kv_attend(s["q"], s["cache"], s["pages"], s["lens"], s["node"], s["parent"], ws=s["ws"])
    lens = vt.vt_kv_commit(s["cache"], s["pages"], s["lens"], s["path"], s["n_accept"])
    return [x for x in s["cache"] if x is not None], lens


# ---- what a pass cannot do without -----------------------------------------------------------------------
def work(case):
    S, Hk, D, kind = case["S"], case["Hk"], case["D"], case["kind"]
    lens = _lengths(case)
    row = 2.0 * Hk * (D + 1 if case["e4m3"] else 2 * D)                         # a token's keys and values in the cache
    if kind == "write":
        T = S * case["rows"] if case["rows"] else sum(lens)
        moved = T * (2.0 * D * (2 * case["Hq"] + 2 * Hk) + row)
        return {"bytes": moved + (T * (row + 4.0 * Hk * D) if case["e4m3"] else 0.0), "flops": 10.0 * T * (case["Hq"] + Hk) * D}
    if kind == "read":
        return {"bytes": sum(lens) * (row + 4.0 * Hk * D + 8.0), "flops": 0.0}
    if kind == "attend":
        Q, Hq = case["Q"], case["Hq"]
        tree = min(case["nodes"], 4 * Q)                                        # nodes that some row sees, about
        seen = sum(lens) + S * tree
        return {"bytes": seen * row + S * Q * Hq * (4.0 * D + 4.0), "flops": 4.0 * Q * Hq * D * seen}
    return {"bytes": 2.0 * S * min(4.0, case["nodes"]) * row, "flops": 0.0}


# ---- the definitions, in 64 bits ---------------------------------------------------------------------------
def _stored64(cache, which, page, place):
    x, e = cache[which], cache[which + 2]
    if e is None:
        return x[page, :, place].to(torch.float64)
    return x.view(torch.uint8)[page, :, place].view(torch.float8_e4m3fn).to(torch.float64) * _power64(e[page, :, place].long() - 127)[..., None]


def _power64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _as_e4m3(x):
    """Rows of 64-bit values as the cache stands for them: three mantissa bits under a power of two that brings the largest to at most 448."""
    big = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(big > 0, big, torch.ones_like(big)) / 448.0) - 1e-13).clamp(min=-126.0)
    y = x / _power64(e)
    ulp = _power64(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)) + 1e-13) - 3.0)
    return torch.round(y / ulp) * ulp * _power64(e)


def exact(case, seed):
    s = prepare(case, seed)
    S, D, page, kind, pages = case["S"], case["D"], case["page"], case["kind"], s["pages"].long()
    if kind == "commit":
        return None                                                             # bits that are moved
    if kind == "attend":
        return _exact_attend(s)
    seq, index = s["seq"].long(), s["index"].long()
    where = pages[seq, index // page], index % page
    if kind == "read":
        return _stored64(s["cache"], 0, *where), _stored64(s["cache"], 1, *where)
    turn = s["positions"].to(torch.float64)[:, None, None] * s["inv_freq"]
    half = case["rot"] // 2

    def rows(x, w):
        x = x.to(torch.float64)
        if w is not None:
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS) * w.to(torch.float64)
        z = torch.polar(torch.ones_like(turn), turn) * torch.complex(x[..., :half].contiguous(), x[..., half: 2 * half].contiguous())
        return torch.cat([z.real, z.imag, x[..., 2 * half:]], -1)

    q, k, v = rows(s["q"], s["qw"]), rows(s["k"], s["kw"]), s["v"].to(torch.float64)
    if case["e4m3"]:
        return q, _as_e4m3(k), _as_e4m3(v)
    ck, cv = (x.to(torch.float64) for x in s["cache"][:2])
    ck[where[0], :, where[1]], cv[where[0], :, where[1]] = k, v
    return q, ck, cv


def _exact_attend(s):
    case, page = s["case"], s["case"]["page"]
    Q, Hq, Hk, D, N = case["Q"], case["Hq"], case["Hk"], case["D"], case["nodes"]
    out = torch.zeros((case["S"], Q, Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.full((case["S"], Q, Hq), -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lengths(case)):
        index = torch.arange(n + N, device=DEV)
        sees = torch.ones((Q, n + N), dtype=torch.bool)
        if N:
            up = s["parent"][b].tolist()
            sees[:, n:] = False
            for r, at in enumerate(s["node"].view(-1, Q)[b].tolist()):
                while at >= 0:
                    sees[r, n + at] = True
                    at = up[at]
        if n + N == 0:
            continue
        where = s["pages"][b].long()[index // page], index % page
        k, v = _stored64(s["cache"], 0, *where), _stored64(s["cache"], 1, *where)
        for h in range(Hq):
            x = s["q"].view(-1, Q, Hq, D)[b, :, h].to(torch.float64) @ k[:, h // (Hq // Hk)].T / D ** 0.5
            x = torch.where(sees.to(DEV), x, torch.full_like(x, -math.inf))
            lse[b, :, h] = torch.logsumexp(x, -1)
            out[b, :, h] = torch.softmax(x, -1) @ v[:, h // (Hq // Hk)]
    return out.reshape(-1, Hq, D), lse.reshape(-1, Hq)
