"""The cache's calls with the head's and the tree's, as a drafting step uses them: every depth writes its rows, attends, and expands; the
draft is reranked and verified, and the accepted path becomes part of the committed tokens."""
import pytest
import torch

import kv_util as ku
import paper_2506_22694_b200 as vt

pytestmark = pytest.mark.gpu
I32 = torch.int32
D, HQ, HK, HID, K, TOPK, DEPTHS, BUDGET = 64, 8, 2, 512, 700, 4, 3, 12
CAP = TOPK + (DEPTHS - 1) * TOPK * TOPK


class Body:
    """A drafter's body of one layer: embedding, projections, the cache's calls, the output projection."""

    def __init__(self, e4m3, page):
        c = lambda shape, seed, std: ku.bf16(shape, seed, std).cuda()
        self.emb, self.qkv, self.o = c((1000, HID), 1, 1.0), c((HID, (HQ + 2 * HK) * D), 2, HID ** -0.5), c((HQ * D, HID), 3, (HQ * D) ** -0.5)
        self.W, self.map = c((K, HID), 4, 0.1), torch.randperm(1000, generator=ku.gen(5))[:K].to(I32).cuda()
        self.qw, self.kw = ((1 + ku.bf16((D,), s, 0.2).float()).to(torch.bfloat16).cuda() for s in (6, 7))
        self.freqs = vt.vt_rope_freqs(D, 10000.0)
        n = -(-(300 + CAP) // page)
        self.cache = vt.kv_cache(n + 1, HK, page, D, e4m3)
        self.pages = torch.randperm(n + 1, generator=ku.gen(8))[:n].to(I32).view(1, n).cuda()
        self.ws = ku.attend_ws(1, TOPK, HQ, HK, D)
        self.head_ws = vt.Workspace(vt.workspace_bytes(vt.VT_OP_DRAFT_HEAD, 0, 0, K, HID, TOPK, TOPK))

    def rows(self, ids, index, positions):
        x = self.emb[ids.long()]
        q, k, v = ((x @ self.qkv).split([HQ * D, HK * D, HK * D], 1))
        one = lambda y: y.view(len(ids), -1, D)
        q = vt.vt_qkv_write(one(q), one(k), one(v), self.cache, self.pages, index, None, positions, self.freqs, self.qw, self.kw, ws=self.ws)
        return x, q

    def hidden(self, ids, index, positions, lens, node, parent):
        x, q = self.rows(ids, index, positions)
        y, _ = vt.vt_kv_attend(q, self.cache, self.pages, lens, node, parent, ws=self.ws)
        return x + y.reshape(len(ids), HQ * D) @ self.o

    def fresh(self, ids):
        """Hidden states of a text's tokens without a cache of drafts: written into a new one, each attending to what is in front of it."""
        n, keep = len(ids), (self.cache, self.pages)
        self.cache = vt.kv_cache(self.cache[0].shape[0], HK, self.cache[0].shape[2], D, self.cache[2] is not None)
        at = torch.arange(n, dtype=I32).cuda()
        x, q = self.rows(ids, at, at)
        out = []
        for i in range(n):
            y, _ = vt.vt_kv_attend(q[i:i + 1], self.cache, self.pages, at[i:i + 1] + 1, ws=self.ws)
            out.append(x[i:i + 1] + y.reshape(1, HQ * D) @ self.o)
        rows = vt.vt_kv_read(self.cache, self.pages, at)
        self.cache, self.pages = keep
        return torch.cat(out), rows


@pytest.mark.parametrize("e4m3,page", [(False, 16), (True, 16), (False, 7), (True, 32)])
def test_draft_verify_commit(e4m3, page):
    body = Body(e4m3, page)
    text = torch.randint(0, 1000, (41,), generator=ku.gen(9)).to(I32).cuda()
    at = torch.arange(40, dtype=I32).cuda()
    body.rows(text[:40], at, at)                                          # the prompt; its last token is drafted from
    temp = torch.ones(TOPK, device="cuda")
    lens = torch.tensor([40], dtype=I32).cuda()
    for step in range(3):
        n = int(lens)
        pool = vt.tree_pool(CAP)
        # the row behind the committed tokens: written in place lens, and attended as the last committed one
        h = body.hidden(text[n:n + 1], lens, lens, lens + 1, None, None)
        now = lens + 1
        _, _, front = vt.vt_draft_head_expand(h, body.W, body.map, temp[:1], TOPK, None, None, pool, 0, TOPK, ws=body.head_ws)
        base, hidden = TOPK, {}
        for depth in range(1, DEPTHS):
            h = body.hidden(pool[0][front.long()], now + front, now + depth - 1 + 0 * front, now, front, pool[1][None])
            hidden.update({int(f): h[i] for i, f in enumerate(front.tolist())})
            _, _, front = vt.vt_draft_head_expand(h, body.W, body.map, temp, TOPK, None, front, pool, base, TOPK, ws=body.head_ws)
            base += TOPK * TOPK
        body.rows(pool[0][front.long()], now + front, now + DEPTHS - 1 + 0 * front)                  # (the last depth's rows, for the commit)
        # every drafted row against the text that its path spells, run from the start
        tok, par = pool[0].tolist(), pool[1].tolist()
        for f, h in hidden.items():
            path, i = [], f
            while i >= 0:
                path.insert(0, tok[i])
                i = par[i]
            want, _ = body.fresh(torch.cat([text[:n + 1], torch.tensor(path, dtype=I32).cuda()]))
            # the same operands in another order of sums: two roundings to bf16 of the attention's output (2^-8 of it each, through a projection of
            # unit gain), and one of the sum
            y = (want[-1] - body.emb[path[-1]]).float()
            assert float((h.float() - want[-1].float()).abs().max()) <= 2.0 ** -7 * float(want[-1].float().abs().max()) + 2.0 ** -6 * float(y.abs().max())
        nodes, token, parent = vt.vt_tree_rerank(pool, base, BUDGET)
        written = set(range(TOPK)) | set(hidden) | set(front.tolist())
        # the target accepts a path whose rows are in the cache
        target = torch.full((1, BUDGET + 1), 5000, dtype=I32)
        cur, taken = -1, []
        while True:
            below = [i for i in range(BUDGET) if parent[i] == cur and int(nodes[i]) in written and int(nodes[i]) in hidden]
            if not below:
                break
            target[0, cur + 1] = token[below[-1]]
            cur = below[-1]
            taken.append(int(token[cur]))
        n_accept, path, emitted = vt.vt_verify_greedy(token.view(1, -1), parent.view(1, -1), target.cuda())
        m = int(n_accept)
        assert m >= 1
        lens = vt.vt_kv_commit(body.cache, body.pages, now, path, n_accept, nodes.view(1, -1), ws=body.ws)
        assert int(lens) == n + 1 + m
        text = torch.cat([text[:n + 1], emitted[0, :m], torch.tensor([17 * step + 3], dtype=I32).cuda()])
        # the committed tokens are those of the text, run from the start
        _, want = body.fresh(text[:n + 1 + m])
        got = vt.vt_kv_read(body.cache, body.pages, torch.arange(n + 1 + m, dtype=I32).cuda())
        for a, b in zip(got, want):
            # projections of other row counts may be summed in another order: a bf16 rounding of the projection (2^-8), which eight bits may round
            # to the neighbouring value (2^-3)
            off = (a.float() - b.float()).abs()
            assert float((off / b.float().abs().clamp(min=2.0 ** -6 * float(b.float().abs().max()))).max()) <= (2.0 ** -2 if e4m3 else 2.0 ** -5)
            assert float((off > 0).float().mean()) < 0.05
    assert body.ws.read_status()[1] == 0
