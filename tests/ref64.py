"""Plain 64-bit implementations that the tests of prompts, page tables and block-scaled
pages compare with (test infrastructure; no code of the package)."""
import numpy as np
import torch


def causal(q, k, v, starts, scale):
    """Causal attention of packed rows, one sequence and head at a time.  Returns the
    outputs, the averages of |v| under the same weights (what a relative error of
    the weights is multiplied by), and per row the largest scale * sum |q_d k_d|."""
    q, k, v = (x.double() for x in (q, k, v))
    N, Hq, D = q.shape
    G = Hq // k.shape[1]
    out = torch.zeros_like(q)
    mag = torch.zeros_like(q)
    top = torch.zeros((N, Hq), dtype=torch.float64, device=q.device)
    for a, b in zip(starts[:-1], starts[1:]):
        n = b - a
        if n == 0:
            continue
        seen = torch.ones((n, n), dtype=torch.bool, device=q.device).tril()
        for h in range(Hq):
            qh, kh, vh = q[a:b, h], k[a:b, h // G], v[a:b, h // G]
            x = (qh @ kh.t().contiguous() * scale).masked_fill(~seen, -np.inf)
            w = torch.exp(x - x.amax(1, keepdim=True))
            w = w / w.sum(1, keepdim=True)
            out[a:b, h] = w @ vh
            mag[a:b, h] = w @ vh.abs()
            top[a:b, h] = (qh.abs() @ kh.abs().t().contiguous()).masked_fill(~seen, 0).amax(1) * scale
    return out, mag, top


def e4m3_round(x):
    """Nearest E4M3 numbers (ties to even, at most 448) of float64 values: three bits
    behind the point, least exponent -6."""
    e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6)))
    step = 2.0 ** (e - 3)
    return np.clip(np.rint(x / step) * step, -448.0, 448.0)


def scale_exponent(amax):
    """Least e with amax <= 448 * 2^e, 0 for nothing, within the format's range."""
    if amax == 0:
        return 0
    e = -200
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return min(max(e, -117), 119)


class Pages:
    """Page tables kept with Python lists, one page at a time."""

    def __init__(self, B, page, max_pages, num_pages):
        self.B, self.page, self.max_pages, self.num_pages = B, page, max_pages, num_pages
        self.free = list(range(num_pages - 1, -1, -1))
        self.held = [[] for _ in range(B)]

    def plan(self, kv, new, rows_per_seq, N):
        """(row starts, slots, positions) of one call; pages as the lists say."""
        need = [-(-(a + n) // self.page) for a, n in zip(kv, new)]
        for b in range(self.B - 1, -1, -1):
            while len(self.held[b]) > need[b]:
                self.free.append(self.held[b].pop())
        for b in range(self.B):
            want = need[b] - len(self.held[b])
            if want > len(self.free):
                break
            for _ in range(max(want, 0)):
                self.held[b].append(self.free.pop())
        starts = [sum(new[:b]) for b in range(self.B + 1)]
        slots, pos = [-1] * N, [-1] * N
        for b in range(self.B):
            for r in range(new[b]):
                i = b * rows_per_seq + r if rows_per_seq else starts[b] + r
                p = kv[b] + r
                pos[i] = p
                if p // self.page < len(self.held[b]):
                    slots[i] = self.held[b][p // self.page] * self.page + p % self.page
        return starts, slots, pos


def write_block(live, live_e, new):
    """One block: live rows (codes' values under 2^live_e), new rows (float64); returns
    the values of all rows' codes and the scale's exponent."""
    x = np.concatenate([live * 2.0 ** live_e, new])
    e = scale_exponent(np.abs(x[np.isfinite(x)]).max(initial=0.0))
    y = x * 2.0 ** -e
    return e4m3_round(np.nan_to_num(y, nan=0.0, posinf=1e9, neginf=-1e9)), e


def tree(q, k, v, kv_len, parent, scale, live):
    """Tree attention of one sequence: q [T][Hq][D], k, v [Hkv][rows][D] with node i's row at
    kv_len + i.  Returns the outputs of the `live` first nodes (the others zero) and the
    averages of |v| under the same weights."""
    q, k, v = (x.double() for x in (q, k, v))
    T, Hq, D = q.shape
    G = Hq // k.shape[0]
    out, mag = torch.zeros_like(q), torch.zeros_like(q)
    if not live:
        return out, mag
    anc = torch.zeros((live, live), dtype=torch.bool)
    for i in range(live):
        if parent[i] >= 0:
            anc[i] = anc[int(parent[i])]
        anc[i, i] = True
    seen = torch.cat((torch.ones((live, kv_len), dtype=torch.bool), anc), 1).to(q.device)
    for h in range(Hq):
        kh, vh = k[h // G, :kv_len + live], v[h // G, :kv_len + live]
        x = (q[:live, h] @ kh.t().contiguous() * scale).masked_fill(~seen, -np.inf)
        w = torch.exp(x - x.amax(1, keepdim=True))
        w = w / w.sum(1, keepdim=True)
        out[:live, h] = w @ vh
        mag[:live, h] = w @ vh.abs()
    return out, mag
