"""Plain 64-bit restatement of the key-value cache's calls (host tensors, token by token), and caches to try them on."""
import math

import torch

import paper_2506_22694_b200 as vt

E4M3 = [s * v for s in (1, -1) for v in [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)]]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def bf16(shape, seed, std=1.0):
    return (torch.randn(shape, generator=gen(seed), dtype=torch.float32) * std).to(torch.bfloat16)


def decode(stored, exps):
    """What a host cache stands for, in 64 bits."""
    if exps is None:
        return stored.double()
    table = torch.tensor(E4M3, dtype=torch.float64)
    u = stored.view(torch.uint8).long()
    table[127], table[255] = 480.0, -480.0
    e = exps.long()
    f = torch.where(e == 255, torch.tensor(math.nan, dtype=torch.float64), torch.pow(torch.tensor(2.0, dtype=torch.float64), (e - 127).double()))
    return table[u] * f[..., None]


def encode_row(x):
    """One row (64-bit values) -> (e4m3 bytes, exponent byte), by searching the table of values: nearest, ties to the even byte."""
    if not bool(torch.isfinite(x).all()):
        return torch.zeros(x.numel(), dtype=torch.uint8), 255
    top, e = float(x.abs().max()), -126
    if top > 0:
        e = max(-126, math.frexp(top / 448.0)[1] - 1)
        while e > -126 and top <= 448.0 * 2.0 ** (e - 1):
            e -= 1
        while top > 448.0 * 2.0 ** e:
            e += 1
    y = x.abs() * 2.0 ** -e
    values = torch.tensor(E4M3[:127], dtype=torch.float64)
    far = (y[:, None] - values).abs()
    best = far.min(1)[0]
    near = far <= best[:, None]
    code = torch.arange(127)
    even = torch.where(near & (code % 2 == 0), code, 1000).min(1)[0]
    odd = torch.where(near, code, 1000).min(1)[0]
    out = torch.where(even < 1000, even, odd)
    return (out + 128 * torch.signbit(x).long()).to(torch.uint8), e + 127


def encode(x):
    rows = [encode_row(r) for r in x.double().reshape(-1, x.shape[-1])]
    return (torch.stack([r[0] for r in rows]).view(x.shape).view(torch.float8_e4m3fn),
            torch.tensor([r[1] for r in rows], dtype=torch.uint8).view(x.shape[:-1]))


class Host:
    """A cache on the host and its copy on the device, pages in a random order; `layout`: order of the stored dims."""

    def __init__(self, S, room, heads, d, page, e4m3, seed, layout="nhpd", std=1.0):
        per = max(1, -(-room // page))
        n = S * per + 2
        self.page, self.e4m3, self.S, self.d, self.heads = page, e4m3, S, d, heads
        self.pages = torch.randperm(n, generator=gen(seed))[: S * per].view(S, per).to(torch.int32)
        k, v = bf16((n, heads, page, d), seed + 1, std), bf16((n, heads, page, d), seed + 2, std)
        self.ke = self.ve = None
        if e4m3:
            self.k, self.ke = self._quick(k)
            self.v, self.ve = self._quick(v)
        else:
            self.k, self.v = k, v
        self.layout = layout

    @staticmethod
    def _quick(x):
        """e4m3 rows under exponents of many sizes (any bytes do for reading)."""
        e = torch.randint(110, 130, x.shape[:-1], generator=gen(x.shape[0]), dtype=torch.int32).to(torch.uint8)
        return (x.float() * 100).clamp(-440, 440).to(torch.float8_e4m3fn), e

    def place(self, s, i):
        return int(self.pages[s, i // self.page]), i % self.page

    def device(self):
        def there(x):
            if x is None:
                return None
            if x.dim() == 3 or self.layout == "nhpd":
                return x.cuda()
            order = [0, 2, 1, 3]                                      # tokens outside heads
            raw = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
            return raw.permute(order).contiguous().cuda().view(x.dtype).permute(order)
        self.pages_dev = self.pages.cuda()
        self.dev = tuple(there(x) for x in (self.k, self.v, self.ke, self.ve))
        return self.dev

    def values(self, s, index):
        """(k, v) [n, heads, d] in 64 bits of places `index` of sequence s."""
        at = torch.as_tensor(index, dtype=torch.int64)
        p, j = self.pages[s].long()[at // self.page], at % self.page
        out = []
        for x, e in ((self.k, self.ke), (self.v, self.ve)):
            if e is None:
                out.append(x[p, :, j].double())
            else:
                out.append(decode(x.view(torch.uint8)[p, :, j], e[p, :, j]))
        return out

    def powers(self, s, index):
        """The values' powers of two [n, heads] (e4m3)."""
        at = torch.as_tensor(index, dtype=torch.int64)
        e = self.ve[self.pages[s].long()[at // self.page], :, at % self.page]
        return torch.pow(torch.tensor(2.0, dtype=torch.float64), (e.long() - 127).double())

    def same(self, dev=None):
        """Whether the device's cache holds the host's bytes."""
        for a, b in zip((self.k, self.v, self.ke, self.ve), dev or self.dev):
            if a is None:
                continue
            b = b.cpu().contiguous()
            a, b = (x.contiguous().view(torch.int16 if a.dtype == torch.bfloat16 else torch.uint8) for x in (a, b))
            if not torch.equal(a, b):
                return False
        return True


def attend(host, q, lens, Q, node=None, parent=None, scale=None):
    """(out, lse, bound of |out's error|, bound of |lse's error|), in 64 bits.

    The bounds: a score is a sum of d products in fp32 (each addition off by at most a step, 2^-23 of the sum of magnitudes so far), an
    exponential by 2^-21, a weight as two bf16 pieces by 2^-17 or (e4m3) as one of f16 by 2^-11, and there, where it is under 2^-14 of the
    largest weight times power, by 2^-25 of that, times a value of 448 at the most; a relative error of the weights moves their mean by at
    most twice that of the mean magnitude; sums over n tokens add n steps of 2^-23; the result is rounded to bf16 (2^-8) and parts are joined with a few more
    exponentials (2^-20 in all)."""
    T, Hq, d = q.shape
    S, g = host.S, Hq // host.heads
    scale = d ** -0.5 if scale is None else scale
    out, lse = torch.zeros(T, Hq, d, dtype=torch.float64), torch.full((T, Hq), -math.inf, dtype=torch.float64)
    tol, tol_l = torch.zeros(T, Hq, d, dtype=torch.float64), torch.zeros(T, Hq, dtype=torch.float64)
    for s in range(S):
        for r in range(Q):
            t = s * Q + r
            seen = list(range(max(0, int(lens[s]))))
            if node is not None:
                f = int(node[t])
                if f < -1:
                    seen = []
                while f >= 0:
                    seen.append(int(lens[s]) + f)
                    up = f - 1 if parent is None else int(parent[s, f])
                    f = up if up < f else -1
            if not seen:
                continue
            k, v = host.values(s, seen)
            for h in range(Hq):
                x = q[t, h].double()
                z = (k[:, h // g] @ x) * scale
                worst = float((k[:, h // g].abs() @ x.abs()).max()) * abs(scale) * (d + 8) * 2.0 ** -23
                m = z.max()
                if m == -math.inf:
                    continue
                p = torch.exp(z - m)
                out[t, h] = (p[:, None] * v[:, h // g]).sum(0) / p.sum()
                lse[t, h] = m + torch.log(p.sum())
                mean = (p[:, None] * v[:, h // g].abs()).sum(0) / p.sum()
                delta = (2.0 ** -11 if host.e4m3 else 2.0 ** -17) + 2.0 ** -20 + worst
                small = 2.0 ** -25 * 448 * len(seen) * float((p * host.powers(s, seen)[:, h // g]).max() / p.sum()) if host.e4m3 else 0.0
                tol[t, h] = 2.0 ** -8 * out[t, h].abs() + (2 * delta + len(seen) * 2.0 ** -23) * mean * (1 + 2.0 ** -7) + small + 1e-37
                tol_l[t, h] = worst + 2.0 ** -20 + len(seen) * 2.0 ** -23 + 2.0 ** -22 * abs(float(lse[t, h]))
    return out, lse, tol, tol_l


def near(got, ref, tol):
    """NaN and infinity where the reference has them, else within the tolerance."""
    got = got.double().cpu()
    same = (torch.isnan(got) & torch.isnan(ref)) | (got == ref)
    ok = same | ((got - ref).abs() <= tol)
    return bool(ok.all()), float(((got - ref).abs() / tol.clamp(min=1e-300))[~same & torch.isfinite(ref)].max()) if bool((~same & torch.isfinite(ref)).any()) else 0.0


def written(host, q, k, v, index, seq, positions, inv_freq, interleaved, qw, kw, eps):
    """vt_qkv_write on the host cache: (q, bound of its error, and of the keys' in a bf16 cache by place)."""
    d = host.d

    def rows(x, w):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
        size = x.abs()
        if inv_freq is None:
            return x, size
        angle = positions.double()[:, None, None] * inv_freq
        c, s, half = torch.cos(angle), torch.sin(angle), len(inv_freq)
        y, z = x.clone(), size.clone()
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        z[..., a] = z[..., b] = size[..., a] + size[..., b]
        return y, z

    # fp32: d / 2 steps for the sum of squares' root, a few for the scaling, sines to 2^-21; then one rounding to bf16
    def bound(y, z):
        return 2.0 ** -8 * y.abs() + z * ((d / 2 + 16) * 2.0 ** -24 + 2.0 ** -21)

    yk, zk = rows(k, kw)
    for t in range(k.shape[0]):
        s, i = int(seq[t]), int(index[t])
        if i < 0 or s < 0 or s >= host.S or i >= host.pages.shape[1] * host.page:
            continue
        p, j = host.place(s, i)
        if p < 0 or p >= host.k.shape[0]:
            continue
        if host.e4m3:
            b, e = encode(yk[t])
            host.k.view(torch.uint8)[p, :, j], host.ke[p, :, j] = b.view(torch.uint8), e
            b, e = encode(v[t])
            host.v.view(torch.uint8)[p, :, j], host.ve[p, :, j] = b.view(torch.uint8), e
        else:
            host.v[p, :, j] = v[t]
    if q is None:
        return None, None, yk, bound(yk, zk)
    yq, zq = rows(q, qw)
    return yq, bound(yq, zq), yk, bound(yk, zk)


def inv_freq(rot, base):
    return torch.tensor([base ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64)


def attend_ws(S, Q, Hq, Hk, d):
    return vt.Workspace(vt.workspace_bytes(vt.VT_OP_KV_ATTEND, n=S, B=Q, K=Hq, V=Hk, d=d))


def tree(S, N, seed, fan=3):
    """Random parents in front of their children, [S, N]."""
    g = gen(seed)
    out = torch.full((S, N), -1, dtype=torch.int32)
    for i in range(1, N):
        lo = max(-1, i - 1 - 4 * fan)
        out[:, i] = torch.randint(lo, i, (S,), generator=g).to(torch.int32)
    return out
