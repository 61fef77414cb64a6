"""Cases of the serving path around the decoding step, in plain form and through the
public entry points: attention over packed prompts, page tables and slot maps, rows
written into 8-bit pages with a scale per block, and tree attention over such pages.

A case is a dict of plain sizes.  Its "kind" names the operator:

  prompt   causal attention over packed prompts of different lengths
  pages    page tables and slot maps: a decoding step's growth and trim, or the
           admission of prompts and the release of finished ones
  write    rows into E4M3 pages with block scales: prompts, or a step's tree rows and
           then the accepted ones of them
  attn     tree attention (one node: a single token) over such pages

An 8-bit page holds E4M3 codes [Hkv][page][D]; each block of `S` rows of a head has one
scale for its keys and one for its values, powers of two held as biased exponents.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"


def listed():
    return [
        # the smallest: one short turn of a conversation, where launches count
        dict(name="prompt_short", kind="prompt", B=1, lo=19, hi=19, lens=0, Hq=32, Hkv=8, D=128, f32=False, fused=True),
        # a server's batch of prompts, from a few words to a few pages, packed
        dict(name="prompt_batch", kind="prompt", B=16, lo=17, hi=2048, lens=3, Hq=32, Hkv=8, D=128, f32=False, fused=True),
        # one long document
        dict(name="prompt_long", kind="prompt", B=1, lo=8192, hi=8192, lens=0, Hq=32, Hkv=8, D=128, f32=False, fused=False),
        # heads without groups, odd lengths
        dict(name="prompt_heads", kind="prompt", B=3, lo=333, hi=1501, lens=1, Hq=40, Hkv=40, D=128, f32=False, fused=False),
        # the fp32 reference configuration, narrow heads
        dict(name="prompt_f32", kind="prompt", B=4, lo=1, hi=513, lens=2, Hq=4, Hkv=2, D=64, f32=True, fused=False),
        # between two forward passes: every sequence takes pages for its tree, then
        # keeps those of the accepted rows
        dict(name="pages_step", kind="pages", B=16, rows=64, lo=512, hi=8192, lens=4, page=64, admit=False),
        # prompts admitted and finished ones released
        dict(name="pages_admit", kind="pages", B=64, rows=0, lo=16, hi=8192, lens=5, page=64, admit=True),
        # a step's rows: all tree nodes, then the accepted ones over them
        dict(name="write_step", kind="write", B=16, rows=64, lo=512, hi=2048, lens=6, Hkv=8, page=64, S=32, prompt=False),
        # packed prompts into empty pages
        dict(name="write_prompts", kind="write", B=8, rows=0, lo=100, hi=8192, lens=7, Hkv=8, page=128, S=64, prompt=True),
        # single tokens, long contexts
        dict(name="attn_token", kind="attn", B=16, T=1, lo=8192, hi=8192, lens=0, Hq=32, Hkv=8, page=64, S=64, ragged=False),
        # a serving batch with trees of their own sizes
        dict(name="attn_trees", kind="attn", B=16, T=64, lo=512, hi=8192, lens=4, Hq=32, Hkv=8, page=64, S=32, ragged=True),
        # one long document being continued
        dict(name="attn_long", kind="attn", B=1, T=64, lo=32768, hi=32768, lens=0, Hq=32, Hkv=8, page=128, S=128, ragged=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "prompt", "pages", "write", "attn", "attn"])
    lens = rng.randint(10, 10 ** 6)
    if kind == "prompt":
        f32 = rng.random() < 0.2
        Hq, Hkv = rng.choice([(2, 2), (4, 2), (8, 1)] if f32 else [(32, 8), (32, 8), (32, 32), (40, 40), (28, 4), (16, 2)])
        B = _log(rng, 1, 32)
        hi = _log(rng, 1, 1024 if f32 else max(64, min(8192, int(math.sqrt(2 ** 31 / (B * Hq))))))
        return dict(kind="prompt", B=B, lo=max(1, hi // rng.choice([1, 3, 50])), hi=hi, lens=lens, Hq=Hq, Hkv=Hkv,
                    D=rng.choice([64, 128, 128]), f32=f32, fused=rng.random() < 0.5)
    if kind == "pages":
        admit = rng.random() < 0.5
        B = _log(rng, 1, 256)
        hi = _log(rng, 100, min(32768, 524288 // B))
        return dict(kind="pages", B=B, rows=0 if admit else rng.randint(1, 128), lo=max(1, hi // 8), hi=hi, lens=lens,
                    page=rng.choice([32, 64, 128]), admit=admit)
    page = rng.choice([32, 64, 128, 256])
    S = rng.choice([s for s in (32, 64, 128) if s <= page])
    if kind == "write":
        prompt = rng.random() < 0.5
        B = _log(rng, 1, 32)
        hi = _log(rng, 32, 65536 // B if prompt else 2048)
        return dict(kind="write", B=B, rows=0 if prompt else rng.choice([1, rng.randint(2, 96)]), lo=max(1, hi // 4), hi=hi,
                    lens=lens, Hkv=rng.choice([1, 4, 8]), page=page, S=S, prompt=prompt)
    B = _log(rng, 1, 32)
    hi = _log(rng, 64, min(32768, 131072 // B))
    Hq, Hkv = rng.choice([(32, 8), (32, 8), (32, 4), (8, 8)])
    return dict(kind="attn", B=B, T=rng.choice([1, 1, rng.randint(2, 64), 64]), lo=max(1, hi // rng.choice([1, 8])), hi=hi,
                lens=lens, Hq=Hq, Hkv=Hkv, page=page, S=S, ragged=rng.random() < 0.5)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _lengths(c):
    """Lengths of the sequences: the case's own, whatever the seed of its values."""
    r = random.Random(c["lens"])
    return [r.randint(c["lo"], c["hi"]) for _ in range(c["B"])]


def _live(c):
    """Live nodes of the trees (attn), accepted nodes (pages, write)."""
    r = random.Random(c["lens"] + 1)
    if c["kind"] == "attn":
        return [r.randint(max(1, c["T"] // 3), c["T"]) if c["ragged"] else c["T"] for _ in range(c["B"])]
    return [min(c["rows"], r.randint(0, 6)) for _ in range(c["B"])]


def _dims(c):
    """Rows a sequence may hold (whole pages) and pages per sequence."""
    n = [a + max(c.get("rows", 0), c.get("T", 0)) for a in _lengths(c)]
    per = -(-max(n) // c["page"])
    return per * c["page"], per


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _starts(v):
    return _i32([sum(v[:k]) for k in range(len(v) + 1)])


def _codes(x, S):
    """Pages of values as E4M3 codes and the scales' exponents, [..., page / S] blocks."""
    b = x.unflatten(2, (-1, S))  # [pages, heads, blocks, S, D]
    m, e = torch.frexp(b.abs().amax((3, 4)).float())
    e = e - 9 + (m > 448 / 512).int()  # the least e with amax <= 448 * 2^e
    return (b.float() * torch.exp2(-e.float())[..., None, None]).to(torch.float8_e4m3fn).flatten(2, 3), (e + 127).to(torch.uint8)


def _pages(c, g, n):
    """Filled 8-bit pages: heads of different magnitude, blocks with outliers."""
    shape = (n, c["Hkv"], c["page"], 128)
    got = []
    for _ in range(2):
        x = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
        x *= torch.exp2(torch.randint(-2, 2, (1, c["Hkv"], 1, 1), generator=g, device=DEV).float()).bfloat16()
        x *= 1 + 3 * (torch.rand((n, c["Hkv"], c["page"], 1), generator=g, device=DEV) < 0.02).bfloat16()
        got.append(_codes(x, c["S"]))
    (k, ks), (v, vs) = got
    return k.view(torch.uint8), v.view(torch.uint8), torch.stack((ks, vs), -1).contiguous()


def _forest(r, T):
    """Breadth-first forest of T nodes: up to 4, 3, 2, 2, ... children."""
    parent, front, d = [], [-1], 0
    while len(parent) < T:
        nxt = []
        for p in front:
            for _ in range((4, 3, 2)[min(d, 2)] if p < 0 else r.randint(1, (4, 3, 2)[min(d, 2)])):
                if len(parent) < T:
                    parent.append(p)
                    nxt.append(len(parent) - 1)
        front, d = nxt, d + 1
    return parent


def _path(r, parent, n):
    """Accepted nodes, ascending, n of them if the tree is that deep."""
    best = [i for i in range(len(parent))]
    a, path = r.choice(best), []
    while a >= 0:
        path.append(a)
        a = parent[a]
    return path[::-1][:n]


def _page_state(c, held_rows, per, g, spare):
    """Page tables with pages for `held_rows`, the rest on the free list."""
    B, page = c["B"], c["page"]
    held = [-(-n // page) for n in held_rows]
    n = B * per + spare
    ids = torch.randperm(n, generator=g, device=DEV).int()
    table = torch.full((B, per), -1, dtype=torch.int32, device=DEV)
    k = torch.arange(per, device=DEV)
    first = _starts(held)
    has = k < _i32(held)[:, None]
    table = torch.where(has, ids[torch.where(has, first[:-1, None] + k, 0)], table)
    free = torch.cat((ids[sum(held):], torch.full((sum(held),), -1, dtype=torch.int32, device=DEV)))
    return dict(table=table.contiguous(), held=_i32(held), free=free.contiguous(), count=_i32([n - sum(held)]), num_pages=n, per=per)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(int(seed) + 1)
    r = random.Random(int(seed) + 2)
    lens = _lengths(c)
    s = dict(c=c, lens=lens, status=torch.zeros(1, dtype=torch.int32, device=DEV))
    if c["kind"] == "prompt":
        dt = torch.float32 if c["f32"] else torch.bfloat16
        Hq, Hkv, D, N = c["Hq"], c["Hkv"], c["D"], sum(lens)
        if c["fused"]:  # views of one projection's output
            x = torch.randn((N, Hq + 2 * Hkv, D), generator=g, device=DEV, dtype=dt)
            s["q"], s["k"], s["v"] = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        else:
            s["q"], s["k"], s["v"] = (torch.randn((N, h, D), generator=g, device=DEV, dtype=dt) for h in (Hq, Hkv, Hkv))
        s.update(start=_starts(lens), N=N, out=torch.empty((N, Hq, D), dtype=dt, device=DEV))
        return s
    page = c["page"]
    L, per = _dims(c)
    if c["kind"] == "pages":
        B = c["B"]
        if c["admit"]:
            s.update(_page_state(c, [0] * B, per, g, 17), kv=_i32([0] * B), new=_i32(lens), none=_i32([0] * B),
                     N=sum(lens), start=_i32([0] * (B + 1)), start2=_i32([0] * (B + 1)))
            return dict(s, slots=_i32([0] * s["N"]), pos=_i32([0] * s["N"]), slots2=_i32([0] * s["N"]), pos2=_i32([0] * s["N"]))
        N = B * c["rows"]
        s.update(_page_state(c, lens, per, g, 17), kv=_i32(lens), new=_i32([c["rows"]] * B),
                 accepted=_i32([min(c["rows"], r.randint(0, 6)) for _ in range(B)]), N=N)
        return dict(s, **{n: torch.zeros((B, c["rows"]), dtype=torch.int32, device=DEV) for n in ("slots", "pos", "slots2", "pos2")})
    if c["kind"] == "write":
        B, Hkv = c["B"], c["Hkv"]
        T = c["rows"]
        s.update(_page_state(c, [L] * B, per, g, 1))
        s["k8"], s["v8"], s["scales"] = _pages(c, g, s["num_pages"])
        rows = sum(lens) if c["prompt"] else B * T
        s.update(k=torch.randn((rows, Hkv, 128), generator=g, device=DEV, dtype=torch.bfloat16),
                 v=torch.randn((rows, Hkv, 128), generator=g, device=DEV, dtype=torch.bfloat16), N=rows)
        p = torch.arange(L, device=DEV)
        slot = (s["table"].long()[:, p // page] * page + p % page).int()  # [B, L]
        if c["prompt"]:
            s["slots"] = slot[p < _i32(lens)[:, None]]
            return s
        t = torch.arange(T, device=DEV)
        s["slots"] = slot.gather(1, (_i32(lens)[:, None] + t).long()).contiguous()
        paths = [_path(r, _forest(r, T), n) for n in _live(c)]
        s["nodes"] = _i32([x + [-1] * (T - len(x)) for x in paths])
        s["slots2"] = torch.where(t < _i32([len(x) for x in paths])[:, None], s["slots"], -1).contiguous()
        return s
    B, T = c["B"], c["T"]
    live = _live(c)
    s.update(_page_state(c, [a + b for a, b in zip(lens, live)], per, g, 1))
    s["k8"], s["v8"], s["scales"] = _pages(c, g, s["num_pages"])
    s.update(q=torch.randn((B, T, c["Hq"], 128), generator=g, device=DEV, dtype=torch.bfloat16), L=L, kv=_i32(lens),
             live=_i32(live), parent=_i32([_forest(r, T) for _ in range(B)]),
             out=torch.empty((B, T, c["Hq"], 128), dtype=torch.bfloat16, device=DEV))
    # as ptd_tree_attention_workspace_bytes says for up to 64 splits: a program keeps one for all its calls
    s["ws"] = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _softmax_values(x, v):
    """Softmax over the last axis of x (overwritten), times v."""
    x -= x.amax(-1, keepdim=True)
    x.exp_()
    return torch.matmul(x, v) / x.sum(-1, keepdim=True)


def _plain_prompt(s):
    c, N, dev = s["c"], s["N"], s["q"].device
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    G, L, start = Hq // Hkv, max(s["lens"]), s["start"].long()
    r = torch.arange(L, device=dev)
    live = r < (start[1:] - start[:-1])[:, None]  # [B, L]
    at = torch.where(live, start[:-1, None] + r, 0)
    q = s["q"][at].float().unflatten(2, (Hkv, G)).permute(0, 2, 3, 1, 4).flatten(2, 3)  # [B, Hkv, G * L, D]
    k = s["k"][at].float().permute(0, 2, 3, 1).contiguous()
    v = s["v"][at].float().transpose(1, 2).contiguous()
    x = torch.matmul(q * (1 / math.sqrt(D)), k).unflatten(2, (G, L))
    x.masked_fill_(~(live[:, None] & (r[:, None] >= r))[:, None, None], -math.inf)
    o = _softmax_values(x.flatten(2, 3), v).unflatten(2, (G, L)).permute(0, 3, 1, 2, 4).flatten(2, 3)  # [B, L, Hq, D]
    i = torch.arange(N, device=dev)
    b = torch.searchsorted(start[1:].contiguous(), i, right=True)
    return o[b, i - start[b]].to(s["q"].dtype)


def _plain_plan(s, kv, new, packed):
    """Pages for kv + new rows of every sequence (the free list's end first, sequence
    by sequence), surplus ones back on the free list in the reverse order; a slot
    (page * page size + row) and a position for each new row."""
    page, n = s["c"]["page"], s["num_pages"]
    table, held, free = s["table"].long(), s["held"].long(), s["free"].long()
    kv, new, count = kv.long(), new.long(), s["count"].long()
    k = torch.arange(s["per"], device=table.device)
    need = (kv + new + page - 1) // page
    back = (held - need).clamp(min=0)
    order = torch.cumsum(back, 0)[:, None] - back[:, None] + k - need[:, None]
    gone = (k >= need[:, None]) & (k < held[:, None])
    total = back.sum()
    to = torch.where(gone, count + total - 1 - order, n)
    free = torch.cat((free, free[:1])).scatter(0, to.flatten(), table.flatten())[:n]
    count = count + total
    grow = (need - held).clamp(min=0)
    upto = torch.cumsum(grow, 0)
    ok = upto <= count
    rank = (upto - grow - held)[:, None] + k
    fresh = ok[:, None] & (k >= held[:, None]) & (k < need[:, None])
    table = torch.where(fresh, free[(count - 1 - rank).clamp(0, n - 1)], table)
    s["held"].copy_(torch.where(ok, need, held))
    s["count"].copy_(count - torch.where(ok, grow, 0).sum())
    s["table"].copy_(table)
    s["free"].copy_(free)
    ends = torch.cumsum(new, 0)
    start = torch.cat((ends[:1] * 0, ends))
    i = torch.arange(s["N"], device=table.device)
    if packed:
        b = torch.searchsorted(ends, i, right=True).clamp(max=len(kv) - 1)
        row = i - start[b]
    else:
        b, row = i // s["c"]["rows"], i % s["c"]["rows"]
    at = kv[b] + row
    p = at // page
    ok = (row < new[b]) & (p < s["held"][b])
    slot = torch.where(ok, table[b, p.clamp(max=s["per"] - 1)] * page + at % page, -1).int()
    return start.int(), slot, torch.where(row < new[b], at, -1).int()


def _plain_write(s, slots, source):
    """Rows of s["k"], s["v"] at the slots (-1: none): each touched block keeps the rows
    before its first new one, takes the least power of two that holds all of them as its
    scale, and is coded anew."""
    S, page, Hkv = s["c"]["S"], s["c"]["page"], s["c"]["Hkv"]
    blocks, dev = page // S, slots.device
    total = s["num_pages"] * blocks
    slot = slots.flatten().long()
    block = torch.where(slot >= 0, slot // S, total)
    first = torch.full((total + 1,), S, device=dev).scatter_reduce(0, block, torch.where(slot >= 0, slot % S, S), "amin")
    touched = torch.unique(block)  # the last may stand for no block
    touched = touched[touched < total]
    line = torch.zeros(total + 1, dtype=torch.long, device=dev).scatter(0, touched, torch.arange(len(touched), device=dev))
    real = slot >= 0
    page_of, block_of = touched // blocks, touched % blocks
    keep = torch.arange(S, device=dev) < first[touched][:, None]  # [touched, S]
    fresh = torch.zeros(keep.shape, dtype=torch.bool, device=dev)
    fresh[line[block[real]], slot[real] % S] = True
    for name, rows, kind in (("k8", s["k"], 0), ("v8", s["v"], 1)):
        code = s[name].view(torch.float8_e4m3fn).unflatten(2, (blocks, S)).transpose(1, 2)  # [pages, blocks, Hkv, S, D]
        e = s["scales"][..., kind].transpose(1, 2)  # [pages, blocks, Hkv]
        old = code[page_of, block_of].float() * torch.exp2(e[page_of, block_of].float() - 127)[..., None, None]
        x = torch.where(keep[:, None, :, None], old, 0)
        x.transpose(1, 2)[line[block[real]], slot[real] % S] = rows[source[real]].float()
        m, e = torch.frexp(x.abs().amax((2, 3)))
        e = torch.where(m > 0, (e - 9 + (m > 448 / 512)).clamp(-117, 119), 0)
        y = (x * torch.exp2(-e.float())[..., None, None]).to(torch.float8_e4m3fn)
        y = torch.where((keep | fresh)[:, None, :, None], y.view(torch.uint8), code.view(torch.uint8)[page_of, block_of])
        s[name].unflatten(2, (blocks, S)).transpose(1, 2)[page_of, block_of] = y
        s["scales"][..., kind].transpose(1, 2)[page_of, block_of] = (e + 127).to(torch.uint8)


def _plain_attn(s):
    c, dev = s["c"], s["q"].device
    B, T, Hq, Hkv, page = c["B"], c["T"], c["Hq"], c["Hkv"], c["page"]
    G, L = Hq // Hkv, s["L"]
    at = s["table"].long().clamp(min=0)

    def rows(codes, kind):  # [B, Hkv, L, D]
        x = codes.view(torch.float8_e4m3fn)[at].float()  # [B, per, Hkv, page, D]
        e = torch.exp2(s["scales"][..., kind][at].float() - 127)  # [B, per, Hkv, blocks]
        x = x.unflatten(3, (-1, c["S"])) * e[..., None, None]
        return x.flatten(3, 4).transpose(1, 2).flatten(2, 3)

    # ancestors: seen through the parent, its parent's, and so on, doubling each time
    up = s["parent"].long()
    t = torch.arange(T, device=dev)
    see = torch.zeros((B, T, T + 1), dtype=torch.bool, device=dev)
    see[:, t, t] = True
    see = torch.cat((see, torch.zeros_like(see[:, :1])), 1)  # node T: none
    up = torch.cat((torch.where(up < 0, T, up), torch.full((B, 1), T, device=dev)), 1)
    for _ in range(max(1, T.bit_length())):
        see = see | see.gather(1, up[..., None].expand(-1, -1, T + 1))
        up = up.gather(1, up)
    kv, live = s["kv"].long(), s["live"].long()
    j = torch.arange(L, device=dev)
    node = (j - kv[:, None]).clamp(0, T - 1)  # [B, L]
    vis = (j < kv[:, None])[:, None] | ((j >= kv[:, None]) & (j < (kv + live)[:, None]))[:, None] & \
        see[:, :T, :T].gather(2, node[:, None].expand(-1, T, -1))  # [B, T, L]
    q = s["q"].float().unflatten(2, (Hkv, G)).permute(0, 2, 3, 1, 4).flatten(2, 3)  # [B, Hkv, G * T, D]
    x = torch.matmul(q * (1 / math.sqrt(128)), rows(s["k8"], 0).transpose(2, 3).contiguous()).unflatten(2, (G, T))
    x.masked_fill_(~vis[:, None, None], -math.inf)
    v = torch.where((j < (kv + live)[:, None])[:, None, :, None], rows(s["v8"], 1), 0)
    o = _softmax_values(x.flatten(2, 3), v).unflatten(2, (G, T)).permute(0, 3, 1, 2, 4).flatten(2, 3)
    return torch.where((t < live[:, None])[..., None, None], o, 0).to(torch.bfloat16)


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _own_prompt(s):
    import paper_2607_10661_amd as P
    c, t = s["c"], P.PTD_F32 if s["c"]["f32"] else P.PTD_BF16
    shape = P.PromptShape(c["B"], s["N"], c["Hq"], c["Hkv"], c["D"], s["q"].stride(0), s["k"].stride(0), s["v"].stride(0), t, t, 0.0)
    P.ptd_prompt_attention(s["q"], s["k"], s["v"], s["start"], s["out"], shape, s["status"])
    return s["out"]


def _own_pages(s):
    import paper_2607_10661_amd as P
    c = s["c"]
    return P.PageState(s["table"].data_ptr(), s["held"].data_ptr(), s["free"].data_ptr(), s["count"].data_ptr(), c["B"],
                       c["page"], s["per"], s["num_pages"])


def _own_blocks(s):
    import paper_2607_10661_amd as P
    c = s["c"]
    return P.KVPagesFp8Blk(s["k8"].data_ptr(), s["v8"].data_ptr(), s["scales"].data_ptr(), s["table"].data_ptr(), c["page"],
                           s["per"], s["num_pages"], c["S"])


def _own_write(s):
    import paper_2607_10661_amd as P
    c, kv = s["c"], _own_blocks(s)
    ld = s["k"].stride(0)
    P.ptd_kv_write_fp8blk(s["k"], s["v"], P.PTD_BF16, ld, ld, s["N"], s["slots"], None, 0, kv, c["Hkv"], 128, s["status"])
    if not c["prompt"]:
        P.ptd_kv_write_fp8blk(s["k"], s["v"], P.PTD_BF16, ld, ld, s["N"], s["slots2"], s["nodes"], c["rows"], kv, c["Hkv"], 128,
                              s["status"])


def _own_attn(s):
    import paper_2607_10661_amd as P
    c = s["c"]
    shape = P.AttnShape(c["B"], c["Hq"], c["Hkv"], 128, s["L"], P.PTD_BF16, P.PTD_BF16, 0.0)
    P.ptd_tree_attention_paged_fp8blk(s["q"], _own_blocks(s), s["kv"], s["live"] if c["ragged"] else None, s["parent"], c["T"],
                                      s["out"], shape, s["ws"], s["ws"].numel(), s["status"])
    return s["out"]


def _plan(s, kv, new, names):
    c = s["c"]
    if own:
        import paper_2607_10661_amd as P
        P.ptd_page_plan(_own_pages(s), kv, new, s["N"], c["rows"], s.get(names[0]), s[names[1]], s[names[2]], s["status"])
        got = [s.get(n) for n in names]
    else:
        got = list(_plain_plan(s, kv, new, c["admit"]))
        got[0] = got[0] if c["admit"] else None
        got[1:] = [x.view_as(s[names[1]]) for x in got[1:]]
    return dict(zip(names, got))


def run(state):
    s, c = state, state["c"]
    if c["kind"] == "prompt":
        return _own_prompt(s) if own else _plain_prompt(s)
    if c["kind"] == "pages":
        out = _plan(s, s["kv"], s["new"], ("start", "slots", "pos"))
        if c["admit"]:
            out.update(_plan(s, s["kv"], s["none"], ("start2", "slots2", "pos2")))
        else:
            out.update(_plan(s, s["kv"], s["accepted"], ("start2", "slots2", "pos2")))
        return dict(out, table=s["table"], held=s["held"], free=s["free"], count=s["count"])
    if c["kind"] == "write":
        if own:
            _own_write(s)
        else:
            i = torch.arange(s["N"], device=s["slots"].device)
            _plain_write(s, s["slots"], i)
            if not c["prompt"]:
                _plain_write(s, s["slots2"], i // c["rows"] * c["rows"] + s["nodes"].flatten().clamp(min=0))
        # the codes as the numbers they stand for, in units of their block's scale
        return dict(k=s["k8"].view(torch.float8_e4m3fn), v=s["v8"].view(torch.float8_e4m3fn), scales=s["scales"])
    return _own_attn(s) if own else _plain_attn(s)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and its outputs in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    c, lens = case, _lengths(case)
    if c["kind"] == "prompt":
        e = 4 if c["f32"] else 2
        return {"bytes": sum(lens) * (2 * c["Hq"] + 2 * c["Hkv"]) * c["D"] * e,
                "flops": 4 * c["Hq"] * c["D"] * sum(n * (n + 1) // 2 for n in lens)}
    if c["kind"] == "pages":
        rows = sum(lens) if c["admit"] else c["B"] * c["rows"]
        pages = sum(-(-n // c["page"]) for n in lens) if c["admit"] else -(-rows // c["page"])
        # slots and positions of both calls, pages taken and given back, lengths
        return {"bytes": 2 * 8 * rows + 4 * 4 * pages + 2 * 16 * c["B"], "flops": 0}
    if c["kind"] == "write":
        rows = sum(lens) if c["prompt"] else c["B"] * c["rows"] + sum(_live(c))
        return {"bytes": rows * (c["Hkv"] * 128 * 2 * 3 + 4), "flops": 0}
    live = _live(c)
    keys = sum(lens) + sum(live)
    return {"bytes": 2 * keys * c["Hkv"] * (128 + 1 / c["S"]) + 2 * sum(live) * c["Hq"] * 128 * 2,
            "flops": 4 * c["Hq"] * 128 * sum(n * k for n, k in zip(live, lens))}


def _exact_rows(q, k, v, vis):
    """softmax(q k / sqrt(D)) v over the visible keys, in 64 bits; vis [rows, keys]."""
    x = (q.double() @ k.double().t().contiguous()) / math.sqrt(q.shape[-1])
    p = torch.softmax(x.masked_fill(~vis, -math.inf), -1)
    return p @ v.double().contiguous()


def _exact_e4m3(x):
    """Nearest E4M3 numbers, ties to even: 3 bits behind the point, least exponent -6."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    c = case
    if c["kind"] == "pages":
        return None
    s = prepare(case, seed)
    lens = s["lens"]
    if c["kind"] == "prompt":
        out = torch.empty(s["out"].shape, dtype=torch.float64, device=DEV)
        at, G = 0, c["Hq"] // c["Hkv"]
        for n in lens:
            see = torch.ones((n, n), dtype=torch.bool, device=DEV).tril()
            for h in range(c["Hq"]):
                out[at:at + n, h] = _exact_rows(s["q"][at:at + n, h], s["k"][at:at + n, h // G], s["v"][at:at + n, h // G], see)
            at += n
        return out
    S, page = c["S"], c["page"]
    table = s["table"].tolist()
    if c["kind"] == "write":
        vals = {n: s[n].view(torch.float8_e4m3fn).double() for n in ("k8", "v8")}
        T = c["rows"]
        calls = [(lens, None)] if c["prompt"] else [([T] * c["B"], None), ([int((x >= 0).sum()) for x in s["nodes"]], s["nodes"].tolist())]
        for counts, nodes in calls:
            row = 0
            for b, n in enumerate(counts):
                at = 0 if c["prompt"] else lens[b]
                src = list(range(row, row + n)) if nodes is None else [b * T + x for x in nodes[b][:n]]
                row += n
                done = 0
                while done < n:
                    r = at + done
                    pg, o = table[b][r // page], r % page
                    blk, off = o // S, o % S
                    m = min(S - off, n - done)
                    sl = slice(blk * S, blk * S + off + m)
                    for kind, (name, rows) in enumerate((("k8", s["k"]), ("v8", s["v"]))):
                        old = vals[name][pg, :, blk * S:blk * S + off] * torch.exp2(s["scales"][pg, :, blk, kind].double() - 127)[:, None, None]
                        x = torch.cat((old, rows[src[done:done + m]].double().transpose(0, 1)), 1)
                        e = torch.ceil(torch.log2(x.abs().amax((1, 2)) / 448))
                        vals[name][pg, :, sl] = _exact_e4m3(x * torch.exp2(-e)[:, None, None])
                        s["scales"][pg, :, blk, kind] = (e + 127).to(torch.uint8)
                    done += m
        return dict(k=vals["k8"], v=vals["v8"], scales=None)
    G = c["Hq"] // c["Hkv"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    parents = s["parent"].tolist()
    for b, (n, m) in enumerate(zip(lens, _live(c))):
        ids = s["table"][b, :-(-(n + m) // page)].long()

        def rows(codes, kind):
            x = codes[ids].view(torch.float8_e4m3fn).double()
            e = torch.exp2(s["scales"][ids][..., kind].double() - 127).repeat_interleave(S, 2)
            return (x * e[..., None]).transpose(0, 1).reshape(c["Hkv"], -1, 128)[:, :n + m]

        k, v = rows(s["k8"], 0), rows(s["v8"], 1)
        anc = [[False] * m for _ in range(m)]
        for i in range(m):
            a = i
            while a >= 0:
                anc[i][a] = True
                a = parents[b][a]
        vis = torch.cat((torch.ones((m, n), dtype=torch.bool), torch.tensor(anc, dtype=torch.bool).view(m, m)), 1).to(DEV)
        for h in range(c["Hq"]):
            out[b, :m, h] = _exact_rows(s["q"][b, :m, h], k[h // G], v[h // G], vis)
    return out
