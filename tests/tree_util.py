"""What the tests of the paged operators share: pools of stored values, and the attention in 64 bits on the host, written from
the definition (Eq. 7 on the stored arrays, soft-max over the keys that are seen) without the library."""
import math

import torch

D = 128


class Pool:
    """Stored pages for `units` units.  Everything is drawn on the host; .encoded(lo, hi) is the device form."""

    def __init__(self, units, pages, page_len, K=16, B=64, T=1, S=1, bits=2, fp8=False, seed=0, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.K, self.B, self.T, self.S, self.bits, self.fp8, self.L, self.pages = K, B, T, S, bits, fp8, page_len, pages
        n = pages * page_len
        self.cent = (spread * torch.randn(units, pages, S, K, D, generator=g)).to(torch.bfloat16)
        self.ids = torch.randint(0, K, (units, n, S), generator=g)
        fields = [0, 1, 3] if bits == 2 else [v & 15 for v in range(-7, 8)]
        pick = torch.tensor(fields)[torch.randint(0, len(fields), (units, n, T, D), generator=g)]
        self.level = torch.where(pick >= 1 << (bits - 1), pick - (1 << bits), pick)
        per = 8 // bits
        self.codes = (pick.view(units, n, T, D // per, per) << (bits * torch.arange(per))).sum(-1).to(torch.uint8)
        if fp8:
            self.scales = torch.randint(0, 52, (units, n, T, D // B), generator=g).to(torch.uint8)       # zero and subnormals too
            e, m = (self.scales >> 3).double(), (self.scales & 7).double()
            self.scale_values = torch.where(e > 0, (1 + m / 8) * torch.exp2(e - 7), m / 8 * 2.0 ** -6)
        else:
            s = spread * torch.rand(units, n, T, D // B, generator=g) * 0.5 / (7 if bits == 4 else 1)
            self.scales = s.to(torch.float16)
            self.scale_values = self.scales.double()

    def decoded(self, unit, page, count):
        """(values, sum of the magnitudes of what they are made of) of a page's first tokens, in 64 bits."""
        at = slice(page * self.L, page * self.L + count)
        rows = torch.stack([self.cent[unit, page, s].double()[self.ids[unit, at, s]] for s in range(self.S)])
        part = self.level[unit, at].double() * self.scale_values[unit, at].repeat_interleave(self.B, -1)
        return rows.sum(0) + part.sum(1), rows.abs().sum(0) + part.abs().sum(1)

    def encoded(self, lo, hi, device="cuda"):
        from paper_2602_02958_amd import binding as B
        cent, ids = self.cent[lo:hi], self.ids[lo:hi].to(B.id_dtype(self.K))
        if self.S == 1:
            cent, ids = cent[:, :, 0], ids[:, :, 0]
        return B.Encoded(cent.contiguous().to(device), ids.contiguous().to(device), self.codes[lo:hi].contiguous().to(device),
                         self.scales[lo:hi].contiguous().to(device), self.L, self.S)


def random_parents(seqs, nodes, seed):
    g = torch.Generator().manual_seed(seed)
    back = torch.randint(1, 6, (seqs, nodes), generator=g)
    return torch.clamp(torch.arange(nodes) - back, min=-1).to(torch.int32)


def plain_mask(parents, nodes=None):
    """(bits [B, N, N] bool, depth [B, N]) by walking up from every node."""
    n, m = parents.shape
    see, depth = torch.zeros(n, m, m, dtype=torch.bool), torch.full((n, m), -1, dtype=torch.int32)
    for b in range(n):
        live = m if nodes is None else max(0, min(m, int(nodes[b])))
        for i in range(m):
            path, j = [], i
            while True:
                p = int(parents[b, j])
                if j >= live or p < -1 or p >= j:
                    path = None
                    break
                path.append(j)
                if p == -1:
                    break
                j = p
            if path is not None:
                see[b, i, path] = True
                depth[b, i] = len(path) - 1
    return see, depth


def bits_of(see):
    """[.., N] bool -> [.., ceil(N / 32)] int32 words."""
    n = see.shape[-1]
    w = -(-n // 32)
    pad = torch.zeros(*see.shape[:-1], w * 32, dtype=torch.int64)
    pad[..., :n] = see.long()
    v = (pad.view(*see.shape[:-1], w, 32) << torch.arange(32)).sum(-1)
    return torch.where(v >= 1 << 31, v - (1 << 32), v).to(torch.int32)


def rotate(x, rope):
    """Interleaved pairs by (cos, sin) [n, d/2, 2]."""
    c, s = rope[..., 0].double(), rope[..., 1].double()
    a, b = x[:, 0::2], x[:, 1::2]
    return torch.stack([a * c - b * s, a * s + b * c], -1).flatten(1)


def reference(q, pool, H, table, kv, k_new, v_new, tail_k, tail_v, tails, nodes, see, rope=None, scale=None):
    """Attention in 64 bits with bounds on what the kernel may be off.  pool: units 0..H-1 are K, H..2H-1 are V.  see [B, N, N].
    Returns out, lse, out_tolerance, lse_tolerance.

    The bounds, with u = 2^-11 (a rounding to binary16) and `mag` the sum of the magnitudes of the parts of a decoded value:
    a decoded key or value has passed at most T + S + 2 roundings to binary16 of partial sums below mag (3 more with the
    rotation, whose result is below sqrt(2) mag), so a score is off by at most
        e = scale * sum |q| mag * R u,  and 2^-20 scale sum |q| mag for the fp32 sums (128 terms, 2^-24 each, and the exponent),
    a weight exp(score) by a factor within exp(+-e), itself rounded to binary16 (u; what falls below 2^-14 of the row's
    scale is off by 2^-25 of it, covered by N 2^-25), and the quotient of two such sums
        |out - exact| <= 2^-8 |out| + (exp(2 e) - 1 + u + R u + 2^-16) E|mag_v|,    |lse - exact| <= e + 2^-20 (1 + |lse|)."""
    n, hq, m, _ = q.shape
    g, u = hq // H, 2.0 ** -11
    scale = 1 / math.sqrt(D) if scale is None else scale
    R = pool.T + pool.S + 2
    out, lse = torch.zeros(n, hq, m, D, dtype=torch.float64), torch.full((n, hq, m), -math.inf, dtype=torch.float64)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(n):
        for h in range(H):
            ks, vs, km, vm = [], [], [], []
            for at in range(0, kv[b], pool.L):
                count = min(pool.L, kv[b] - at)
                page = min(max(int(table[b][at // pool.L]), 0), pool.pages - 1)
                x, mag = pool.decoded(h, page, count)
                if rope is not None:
                    x, mag = rotate(x, rope[at:at + count]), 1.5 * (mag[:, 0::2] + mag[:, 1::2]).repeat_interleave(2, 1)
                ks.append(x), km.append(mag)
                x, mag = pool.decoded(H + h, page, count)
                vs.append(x), vm.append(mag)
            for t in (tail_k[b, h, :tails[b]], k_new[b, h, :nodes[b]]):
                ks.append(t.double()), km.append(t.double().abs())
            for t in (tail_v[b, h, :tails[b]], v_new[b, h, :nodes[b]]):
                vs.append(t.double()), vm.append(t.double().abs())
            K, V, km, vm = (torch.cat(t) for t in (ks, vs, km, vm))
            old = kv[b] + tails[b]
            for i in range(nodes[b]):
                seen = torch.cat([torch.ones(old, dtype=torch.bool), see[b, i, :nodes[b]]])
                if not seen.any():
                    continue
                for j in range(g):
                    r = h * g + j
                    qq = q[b, r, i].double()
                    s = scale * (K[seen] @ qq)
                    e = float(scale * (km[seen] @ qq.abs()).max()) * ((R + (3 if rope is not None else 0)) * u + 2.0 ** -20)
                    z = torch.logsumexp(s, 0)
                    w = torch.exp(s - z)
                    out[b, r, i], lse[b, r, i] = w @ V[seen], z
                    spread = w @ vm[seen]
                    tol[b, r, i] = 2.0 ** -8 * out[b, r, i].abs() + (math.expm1(2 * e) + u + R * u + 2.0 ** -16) * spread
                    ltol[b, r, i] = e + 2.0 ** -20 * (1 + abs(float(z)))
    return out, lse, tol, ltol
