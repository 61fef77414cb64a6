"""Plain 64-bit implementations that the tests of query/key norms, token log probabilities
and shared pages compare with (test infrastructure; no code of the package)."""
import math

import torch


def heads(x, weight, positions, inv_freq, rot, interleaved, eps):
    """Norm (eps None: none) and rotation of x [N][H][D].  Returns the outputs and, per element, the
    magnitude that fp32 errors of the rotation scale with: |u| + |v| of the element's pair."""
    x = x.double()
    if eps is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        if weight is not None:
            x = x * weight.double()
    y, mag = x.clone(), x.abs()
    for p in range(rot // 2):
        a, b = (2 * p, 2 * p + 1) if interleaved else (p, p + rot // 2)
        t = (positions.double() * inv_freq[p])[:, None]
        c, s = torch.cos(t), torch.sin(t)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., a] * s + x[..., b] * c
        mag[..., a] = mag[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, mag


def logprobs(row, temperature, token, k):
    """One row of logits: (log probability of the token, entropy, best k indices, their log
    probabilities, and bounds of the absolute errors of the first, the entropy and the last).

    Bounds, with u = 2^-24: a term e^d has a relative error of 3 u |d| from its argument (a
    difference, a product, the rounded scale), 6 u more where the argument is taken from a reference up to 8
    doublings below the largest entry (8 ln 2 < 6), and 4 u from the exponential; up to 129
    terms of a thread (16 chunks of 8, an edge) and 6 steps of a wave are added in fp32, u each; sums go on from
    a larger reference up to 3 times, a factor (4 u) and a product each; the rest is fp64, and the result is rounded to
    fp32."""
    x = row.double()
    V = x.numel()
    order = sorted(range(V), key=lambda i: (-x[i].item(), i))[:k] if V <= 2000 else \
        torch.sort(x, descending=True, stable=True).indices[:k].tolist()
    m = x.max()
    if m == -math.inf:
        return -math.inf, 0.0, order, [-math.inf] * k, 0.0, 0.0
    d = (x - m) / temperature
    e = torch.exp(d)
    live = e > 0
    total = e.sum()
    lse = torch.log1p((x == m).sum().double() - 1 + e[x != m].sum())
    dl = torch.where(live, d, 0.0)
    weighted = (e * dl).sum()
    u = 2.0 ** -24
    term = 3 * u * (dl.abs() + 6) + 4 * u + (129 + 6 + 3 * 5) * u
    rest = torch.where(x != m, e * term, 0.0).sum()  # absolute error of the sum
    e_lse = rest / total
    e_w = (e * dl.abs() * (term + 2 * u)).sum()
    ent = lse - weighted / total
    e_ent = e_lse + e_w / total + weighted.abs() / total * rest / total + u * ent.abs() + 1e-13
    lp = lambda i: (d[i] - lse).item()  # noqa: E731
    top = [lp(i) for i in order]
    got = lp(token) if token is not None else 0.0
    return got, ent.item(), order, top, e_lse.item() + 1e-13, e_ent.item()


class SharedPages:
    """Page tables whose pages several sequences hold, kept with Python lists."""

    def __init__(self, B, page, max_pages, num_pages):
        self.B, self.page, self.max_pages, self.num_pages = B, page, max_pages, num_pages
        self.free = list(range(num_pages - 1, -1, -1))
        self.held = [[] for _ in range(B)]

    def refs(self):
        n = [0] * self.num_pages
        for h in self.held:
            for p in h:
                n[p] += 1
        return n

    def plan(self, kv, new, rows_per_seq, N):
        need = [-(-(a + n) // self.page) for a, n in zip(kv, new)]
        refs = self.refs()
        for b in range(self.B - 1, -1, -1):
            while len(self.held[b]) > need[b]:
                p = self.held[b].pop()
                refs[p] -= 1
                if refs[p] == 0:
                    self.free.append(p)
        status = 0
        for b in range(self.B):
            want = need[b] - len(self.held[b])
            if want > len(self.free):
                status = 12
                break
            for _ in range(max(want, 0)):
                self.held[b].append(self.free.pop())
        refs = self.refs()
        starts = [sum(new[:b]) for b in range(self.B + 1)]
        slots, pos = [-1] * N, [-1] * N
        for b in range(self.B):
            for r in range(new[b]):
                i = b * rows_per_seq + r if rows_per_seq else starts[b] + r
                p = kv[b] + r
                pos[i] = p
                if p // self.page < len(self.held[b]):
                    if refs[self.held[b][p // self.page]] > 1:
                        status = status or 10
                    else:
                        slots[i] = self.held[b][p // self.page] * self.page + p % self.page
        return starts, slots, pos, status

    def fork(self, frm, length):
        """(copy_src, copy_dst, copy_rows); None if there are too few pages."""
        before = self.refs()
        whole = [[] if a < 0 else self.held[a][:n // self.page] for a, n in zip(frm, length)]
        part = [None if a < 0 or n % self.page == 0 else self.held[a][n // self.page] for a, n in zip(frm, length)]
        full = {p for w in whole for p in w}
        src, dst, rows = [-1] * self.B, [-1] * self.B, [0] * self.B
        free, kept = list(self.free), set()
        for b in range(self.B):
            p = part[b]
            if p is None:
                continue
            if p not in full and p not in kept:
                kept.add(p)
                whole[b] = whole[b] + [p]
                continue
            if not free:
                return None
            q = free.pop()
            whole[b] = whole[b] + [q]
            src[b], dst[b], rows[b] = p, q, length[b] % self.page
        self.held, self.free = whole, free
        after = self.refs()
        self.free += [p for p in range(self.num_pages - 1, -1, -1) if before[p] and not after[p]]
        return src, dst, rows

    def compact(self):
        live = sorted({p for h in self.held for p in h})
        n = len(live)
        holes = [p for p in range(n) if p not in set(live)]
        movers = [p for p in live if p >= n]
        to = dict(zip(movers, holes))
        self.held = [[to.get(p, p) for p in h] for h in self.held]
        self.free = list(range(self.num_pages - 1, n - 1, -1))
        pad = [-1] * (self.num_pages // 2 - len(movers))
        return movers + pad, holes + pad
