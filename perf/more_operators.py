"""Cases of serving several samples of one prompt, in plain form and through the public
entry points: norms of queries and keys with the rotation, log probabilities of given
tokens, and pages that sequences share.

A case is a dict of plain sizes.  Its "kind" names the operator:

  qk       norm of every query and key head, rotation by the rows' positions, rows into
           the caches' pages
  logp     log probabilities of given tokens, entropy and the likeliest tokens: of all
           rows of logits, or of the rows along accepted paths
  fork     samples begun from prompts (or beams that continue others): page tables that share
           pages, copies of last pages, the pages of the next rows
  compact  sequences that finish, live pages moved to the front, sequences that begin

A page holds [Hkv][page][128] numbers; `refs` counts the sequences that hold a page.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"


def listed():
    return [
        # the smallest: the next token of one sequence, where launches count
        dict(name="qk_token", kind="qk", B=1, rows=1, lo=4000, hi=4000, lens=0, Hq=32, Hkv=8, D=128, rot=128, inter=False,
             norm=True, f32=False, fused=True, store=True, page=64),
        # a step's draft trees, their rows into pages
        dict(name="qk_trees", kind="qk", B=16, rows=64, lo=512, hi=8192, lens=4, Hq=32, Hkv=8, D=128, rot=128, inter=False,
             norm=True, f32=False, fused=True, store=True, page=64),
        # packed prompts of a batch (their rows go to 8-bit pages afterwards), half of a head turned
        dict(name="qk_prompts", kind="qk", B=8, rows=0, lo=100, hi=8192, lens=7, Hq=32, Hkv=8, D=128, rot=64, inter=False,
             norm=True, f32=False, fused=True, store=False, page=64),
        # the fp32 reference configuration: narrow heads, neighbouring dimensions turned, rotation alone
        dict(name="qk_f32", kind="qk", B=4, rows=0, lo=1, hi=513, lens=2, Hq=4, Hkv=2, D=64, rot=64, inter=True,
             norm=False, f32=True, fused=False, store=True, page=600),
        # one emitted token of one sequence and its alternatives
        dict(name="logp_token", kind="logp", B=1, T=0, V=128256, k=16, f32=False, odd=0, masked=0, tau=1.0, path=False),
        # the emitted tokens of a step of 16 trees: the few rows along the accepted paths
        dict(name="logp_path", kind="logp", B=16, T=64, V=128256, k=5, f32=False, odd=0, masked=0, tau=1.0, path=True),
        # every row of a prompt's logits scored
        dict(name="logp_rows", kind="logp", B=1040, T=0, V=128256, k=5, f32=False, odd=0, masked=0, tau=1.0, path=False),
        # single precision, rows at odd addresses, all but some tokens masked, a low temperature
        dict(name="logp_masked", kind="logp", B=97, T=0, V=32003, k=8, f32=True, odd=1, masked=400, tau=0.7, path=False),
        # two samples of one short prompt, a small model
        dict(name="fork_two", kind="fork", B=2, lo=90, hi=90, lens=0, groups=1, page=64, Hkv=2, layers=2, f8=False, beams=False, rows=1),
        # prompts of a batch, eight samples each, trees of 64 rows next
        dict(name="fork_samples", kind="fork", B=32, lo=512, hi=8192, lens=4, groups=4, page=64, Hkv=8, layers=16, f8=True,
             beams=False, rows=64),
        # beams: every one continues some beam, then gets one token
        dict(name="fork_beams", kind="fork", B=64, lo=1024, hi=4096, lens=5, groups=8, page=32, Hkv=8, layers=16, f8=False,
             beams=True, rows=1),
        # half of a batch finishes, the rest is moved together, others begin; twice
        dict(name="compact", kind="compact", B=64, lo=256, hi=4096, lens=6, page=64, Hkv=8, layers=4, f8=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["qk", "qk", "qk", "logp", "logp", "logp", "fork", "fork", "compact"])
    lens = rng.randint(10, 10 ** 6)
    if kind == "qk":
        f32 = rng.random() < 0.25
        D = rng.choice([64, 128, 128])
        Hq, Hkv = rng.choice([(4, 2), (16, 2), (28, 4), (7, 1)] + ([(32, 8), (32, 32), (40, 40)] if D == 128 else []))
        B = _log(rng, 1, 64)
        rows = rng.choice([0, 1, rng.randint(2, 96)])
        hi = _log(rng, 1, max(2, 1000000 // (B * (Hq + Hkv) * (2 if f32 else 1)))) if not rows else _log(rng, 1, 100000)
        return dict(kind="qk", B=B, rows=rows, lo=max(1, hi // rng.choice([1, 3, 50])), hi=hi, lens=lens, Hq=Hq, Hkv=Hkv, D=D,
                    rot=rng.choice([D, D, D // 2, 16]), inter=rng.random() < 0.3, norm=rng.random() < 0.75, f32=f32,
                    fused=rng.random() < 0.5, store=rng.random() < 0.6, page=rng.choice([32, 64, 100, 256]))
    if kind == "logp":
        f32, path = rng.random() < 0.3, rng.random() < 0.4
        V = rng.choice([_log(rng, 20, 262144), rng.choice([1000, 32000, 128256])])
        B = _log(rng, 1, 64) if path else _log(rng, 1, max(2, min(8192, 60000000 // V)))
        T = rng.randint(1, max(1, min(96, 60000000 // (V * B)))) if path else 0
        return dict(kind="logp", B=B, T=T, V=V, k=rng.choice([0, 1, rng.randint(2, 16)]), f32=f32,
                    odd=rng.choice([0, 0, 1, 5]), masked=rng.choice([0, 0, 50, 1000]), tau=rng.choice([1.0, 1.0, 0.3, 2.0]), path=path)
    page = rng.choice([32, 64, 128])
    f8 = rng.random() < 0.5
    if kind == "fork":
        groups = _log(rng, 1, 8)
        B = groups * _log(rng, 2, 16)
        hi = _log(rng, 10, 8192)
        return dict(kind="fork", B=B, lo=max(1, hi // 8), hi=hi, lens=lens, groups=groups, page=page, Hkv=rng.choice([1, 2, 4, 8]),
                    layers=rng.randint(1, 8), f8=f8, beams=rng.random() < 0.5, rows=rng.choice([1, rng.randint(2, 96)]))
    B = _log(rng, 2, 64)
    hi = _log(rng, 20, 131072 // B)
    return dict(kind="compact", B=B, lo=max(1, hi // 8), hi=hi, lens=lens, page=page, Hkv=rng.choice([1, 4, 8]),
                layers=rng.randint(1, 4), f8=f8)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
EPS, THETA = 1e-6, 500000.0


def _lengths(c, n=None):
    """Lengths of the sequences: the case's own, whatever the seed of its values."""
    r = random.Random(c["lens"])
    return [r.randint(c["lo"], c["hi"]) for _ in range(n or c["B"])]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _paths(c, r):
    """Accepted nodes of each tree: ascending ids, some trees accept nothing."""
    return [sorted(r.sample(range(c["T"]), min(c["T"], r.choice([0, 1, 2, 3, 4, 6])))) for _ in range(c["B"])]


def _prepare_qk(c, g, s):
    lens = _lengths(c)
    at = [(b, p) for b, n in enumerate(lens) for p in (range(n, n + c["rows"]) if c["rows"] else range(n))]
    N, Hq, Hkv, D = len(at), c["Hq"], c["Hkv"], c["D"]
    dt = torch.float32 if c["f32"] else torch.bfloat16
    if c["fused"]:  # views of one projection's output
        x = torch.randn((N, Hq + 2 * Hkv, D), generator=g, device=DEV, dtype=dt)
        x[:, :Hq + Hkv] *= torch.exp(torch.randn((1, Hq + Hkv, 1), generator=g, device=DEV)).to(dt)
        s["q"], s["k"], s["v"] = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    else:
        s["q"], s["k"], s["v"] = (torch.randn((N, h, D), generator=g, device=DEV, dtype=dt) for h in (Hq, Hkv, Hkv))
    s.update(N=N, pos=_i32([p for _, p in at]), q_out=torch.empty((N, Hq, D), dtype=dt, device=DEV),
             k_out=torch.empty((N, Hkv, D), dtype=dt, device=DEV))
    s["wq"], s["wk"] = ((1 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dt) for _ in range(2)) if c["norm"] else (None, None)
    if c["store"]:
        # the rows' pages in any order, a few of others between them
        page = c["page"]
        used = sorted({(b, p // page) for b, p in at})
        n = len(used) + 2
        ids = dict(zip(used, torch.randperm(n, generator=g, device=DEV).tolist()))
        s["slots"] = _i32([ids[b, p // page] * page + p % page for b, p in at])
        s["num_pages"] = n
        s["kp"], s["vp"] = (torch.zeros((n, Hkv, page, D), dtype=dt, device=DEV) for _ in range(2))
    return s


def _prepare_logp(c, g, s):
    r = random.Random(c["V"] * 7 + c["B"])
    R, V, k = c["B"] * (c["T"] + 1), c["V"], min(c["k"], c["V"])
    dt = torch.float32 if c["f32"] else torch.bfloat16
    wide = torch.empty((R, V + c["odd"]), dtype=dt, device=DEV)
    wide.normal_(0.0, 2.0, generator=g)
    x = wide[:, :V]
    # rows from flat to nearly decided: one entry of each row is raised, by 0 to 24
    top = torch.randint(V, (R, 1), generator=g, device=DEV)
    x.scatter_(1, top, (torch.rand((R, 1), generator=g, device=DEV) * 24).to(dt))
    if c["masked"]:  # all but about that many entries are taken out of the distribution
        step = max(1, V // c["masked"])
        keep = torch.arange(V, device=DEV) % step == torch.randint(step, (R, 1), generator=g, device=DEV)
        keep.scatter_(1, top, True)
        x.masked_fill_(~keep, -math.inf)
    # the given tokens: the raised entry, or any (a masked one among them)
    tokens = torch.where(torch.rand((R, 1), generator=g, device=DEV) < 0.6, top, torch.randint(V, (R, 1), generator=g, device=DEV))
    tokens = tokens.view(R).int()
    s.update(R=R, x=x, ld=V + c["odd"], k=k, nodes=None)
    if c["path"]:
        paths = _paths(c, r)
        T = c["T"]
        s["nodes"] = _i32([p + [-1] * (T - len(p)) for p in paths])
        live = torch.arange(T + 1, device=DEV) <= _i32([len(p) for p in paths])[:, None]
        tokens = torch.where(live.view(-1), tokens, -1)
    s["tokens"] = tokens
    f = dict(dtype=torch.float32, device=DEV)
    s.update(logprob=torch.empty(R, **f), entropy=torch.empty(R, **f), idx=torch.empty((R, k), dtype=torch.int32, device=DEV),
             val=torch.empty((R, k), **f))
    # a program keeps one workspace for all its calls
    s["ws"] = torch.empty(R * 64 * (32 + 16 * 16) if R < 4096 else 64 << 20, dtype=torch.uint8, device=DEV)
    return s


def _pages_of(c, g, n, s):
    """Every layer's keys and values: [layers, 2, pages, Hkv, page, 128], and for 8 bits the
    exponents of the scales of 32 rows, [layers, pages, Hkv, page / 32, 2]."""
    shape = (c["layers"], 2, n, c["Hkv"], c["page"], 128)
    if not c["f8"]:
        s["kv"] = torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
        return s
    s["kv"] = torch.randint(0, 0x70, shape, generator=g, device=DEV, dtype=torch.uint8)
    s["scales"] = torch.randint(110, 130, (c["layers"], n, c["Hkv"], c["page"] // 32, 2), generator=g, device=DEV, dtype=torch.uint8)
    return s


def _prepare_fork(c, g, r, s):
    B, page, n = c["B"], c["page"], c["groups"]
    group = B // n
    lens = _lengths(c, n)
    lens = [lens[b // group] for b in range(B)]  # samples of one prompt are of one length
    per = -(-(max(lens) + c["rows"]) // page)
    need = [-(-a // page) for a in lens]
    num = sum(need[::group]) + B * (2 + -(-c["rows"] // page)) + 3
    ids = torch.randperm(num, generator=g, device=DEV).int().tolist()
    table, held, refs, at = [], [], [0] * num, 0
    first = {}
    for b in range(B):
        lead = b // group * group
        if b == lead:  # a prompt's own pages
            row, at = ids[at:at + need[b]], at + need[b]
            first[lead] = row
        elif c["beams"]:  # a beam shares the full pages and has a last page of its own
            row = list(first[lead])
            if lens[b] % page:
                row[-1], at = ids[at], at + 1
        else:
            row = []
        for p in row:
            refs[p] += 1
        table.append(row + [-1] * (per - len(row)))
        held.append(len(row))
    # which sequence each one continues: the prompt, or some beam of its group
    frm = [b // group * group + (r.randrange(group) if c["beams"] else 0) for b in range(B)]
    s.update(per=per, num_pages=num, table=_i32(table), held=_i32(held), refs=_i32(refs), free=_i32(ids[at:] + [-1] * at),
             count=_i32([num - at]), frm=_i32(frm), len=_i32(lens), new=_i32([c["rows"]] * B), none=_i32([0] * B), N=B * c["rows"],
             back=_i32([b if b % group == 0 or c["beams"] else -1 for b in range(B)]),
             next=_i32([[-1] * per] * B), held2=_i32([0] * B), slots=_i32([0] * (B * c["rows"])), pos=_i32([0] * (B * c["rows"])))
    for i in (1, 2):
        s.update({x + str(i): _i32([0] * B) for x in ("src", "dst", "rows")})
    return _pages_of(c, g, num, s)


def _prepare_compact(c, g, r, s):
    B, page = c["B"], c["page"]
    lens = _lengths(c)
    need = [-(-a // page) for a in lens]
    per, num = max(need), sum(need) + 5
    ids = torch.randperm(num, generator=g, device=DEV).int().tolist()
    table, at = [], 0
    for n in need:
        table.append(ids[at:at + n] + [-1] * (per - n))
        at += n
    refs = [0] * num
    for p in ids[:at]:
        refs[p] = 1
    s.update(per=per, num_pages=num, table=_i32(table), held=_i32(need), refs=_i32(refs), free=_i32(ids[at:] + [-1] * at),
             count=_i32([num - at]), len=_i32(lens), none=_i32([0] * B), N=0,
             half=[_i32([a if b % 2 == i else 0 for b, a in enumerate(lens)]) for i in (0, 1)], start=_i32([0] * (B + 1)), slots=_i32([0]),
             moves=[[_i32([0] * max(1, num // 2)) for _ in range(2)] for _ in range(2)])
    return _pages_of(c, g, num, s)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(int(seed) + 1)
    r = random.Random(int(seed) + 2)
    s = dict(c=c, status=torch.zeros(1, dtype=torch.int32, device=DEV))
    if c["kind"] == "qk":
        return _prepare_qk(c, g, s)
    if c["kind"] == "logp":
        return _prepare_logp(c, g, s)
    return _prepare_fork(c, g, r, s) if c["kind"] == "fork" else _prepare_compact(c, g, r, s)


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _turned(x, w, pos, c):
    """Norm over each head, times w; the first `rot` dimensions turned by the positions."""
    x, rot = x.float(), c["rot"]
    if c["norm"]:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    p = torch.arange(rot // 2, device=x.device, dtype=torch.float64)
    a = (pos.double()[:, None] * THETA ** (-2.0 * p / rot))[:, None]  # angles of far positions: 64 bits
    cos, sin = torch.cos(a).float(), torch.sin(a).float()
    if c["inter"]:
        u, v = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack((u * cos - v * sin, u * sin + v * cos), -1).flatten(-2)
    else:
        u, v = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat((u * cos - v * sin, u * sin + v * cos), -1)
    return torch.cat((y, x[..., rot:]), -1)


def _plain_qk(s):
    c = s["c"]
    s["q_out"].copy_(_turned(s["q"], s["wq"], s["pos"], c))
    s["k_out"].copy_(_turned(s["k"], s["wk"], s["pos"], c))
    if c["store"]:
        pg, row = s["slots"].long() // c["page"], s["slots"].long() % c["page"]
        s["kp"][pg, :, row] = s["k_out"]
        s["vp"][pg, :, row] = s["v"]


def _ordered(x):
    """Whole numbers in the order of x's values, -0 as +0."""
    i = (x + 0.0).view(torch.int32).long()
    return torch.where(i < 0, -(i & 0x7FFFFFFF), i)


def _plain_logp(s):
    c, k = s["c"], s["k"]
    live = s["tokens"] >= 0
    if c["path"]:
        T = c["T"]
        row = torch.cat((torch.full_like(s["nodes"][:, :1], -1), s["nodes"]), 1).long() + 1
        row = (row + torch.arange(c["B"], device=row.device)[:, None] * (T + 1)).view(-1)
        at = live.nonzero()[:, 0]
        x = s["x"][row[at]].float()
    else:
        at, x = torch.arange(s["R"], device=live.device), s["x"].float()
    if k:
        # value descending, equal values by the lower index
        key = _ordered(x) * 2 ** 20 + (2 ** 20 - 1 - torch.arange(c["V"], device=x.device))
        idx = torch.topk(key, k, 1).indices
    m = x.amax(1, keepdim=True)
    d = (x - m) * (1.0 / c["tau"])
    e = torch.exp(d)
    total = e.double().sum(1, keepdim=True)  # (a decided row's sum is a one and what is far below it)
    lse = torch.log(total)
    weighted = (e * d.clamp(min=-1e30)).double().sum(1, keepdim=True)

    def put(out, what, none):
        out.fill_(none)
        out[at] = what.to(out.dtype)

    put(s["logprob"], (d.gather(1, s["tokens"][at].long()[:, None]).double() - lse)[:, 0], 0)
    put(s["entropy"], (lse - weighted / total)[:, 0], 0)
    if k:
        put(s["idx"], idx, -1)
        put(s["val"], d.gather(1, idx).double() - lse, 0)


def _plain_fork(s, table, held, frm, nxt, held2, src, dst, rows):
    """Sequence b of the next table holds the first len[b] rows of sequence frm[b] (-1: none):
    whole pages shared; a page that is partly filled stays with the lowest b that goes on in it, if
    no sequence holds it as a whole one, the others get pages of their own for copies.
    Pages that nobody holds any more go back to the list, higher ids first."""
    page, n, per = s["c"]["page"], s["num_pages"], s["per"]
    B = frm.numel()
    a, ln = frm.long().clamp(min=0), torch.where(frm < 0, 0, s["len"]).long()
    old, free, count, refs = table.long(), s["free"].long(), s["count"].long(), s["refs"].long()
    i, k = torch.arange(B, device=old.device), torch.arange(per, device=old.device)
    full, part = ln // page, ln % page > 0
    row = old[a]
    whole = k < full[:, None]
    shared = torch.zeros(n + 1, dtype=torch.long, device=old.device)
    shared.scatter_add_(0, torch.where(whole, row, n).flatten(), torch.ones(B * per, dtype=torch.long, device=old.device))
    last = torch.where(part, row.gather(1, full.clamp(max=per - 1)[:, None])[:, 0], n)
    shared[n] = 0
    lowest = torch.full((n + 1,), B, device=old.device).scatter_reduce(0, last, i, "amin")
    keep = part & (shared[last] == 0) & (lowest[last] == i)
    copy = part & ~keep
    rank = torch.cumsum(copy, 0) - copy.long()
    fresh = free[(count - 1 - rank).clamp(0, n - 1)]
    mine = torch.where(keep, last, torch.where(copy, fresh, n))
    now = shared.scatter_add(0, mine, part.long())[:n]
    gone = (refs > 0) & (now == 0)
    count = count - copy.sum()
    place = torch.where(gone, count + gone.sum() - torch.cumsum(gone, 0), n)
    s["free"].copy_(torch.cat((free, free[:1])).scatter(0, place, torch.arange(n, device=old.device))[:n])
    s["count"].copy_(count + gone.sum())
    s["refs"].copy_(now)
    nxt.copy_(torch.where(whole, row, torch.where(part[:, None] & (k == full[:, None]), mine[:, None], nxt.long())))
    held2.copy_(full + part)
    src.copy_(torch.where(copy, last, -1))
    dst.copy_(torch.where(copy, fresh, -1))
    rows.copy_(torch.where(copy, ln % page, 0))


def _plain_plan(s, table, held, kv, new):
    """Pages for kv + new rows of every sequence: surplus ones are given up, and one that
    nobody holds any more goes back to the list (in the place of the lowest sequence that gave it up, the
    list's order the reverse of theirs); missing ones from the list's end.  A slot for each new row."""
    c, page, n, per = s["c"], s["c"]["page"], s["num_pages"], s["per"]
    B = kv.numel()
    old, free, refs, count = table.long(), s["free"].long(), s["refs"].long(), s["count"].long()
    kv, new, have = kv.long(), new.long(), held.long()
    k, b = torch.arange(per, device=old.device), torch.arange(B, device=old.device)
    need = (kv + new + page - 1) // page
    gone = (k >= need[:, None]) & (k < have[:, None])
    at = torch.where(gone, old, n)
    gave = torch.zeros(n + 1, dtype=torch.long, device=old.device).scatter_add_(0, at.flatten(), gone.flatten().long())
    lowest = torch.full((n + 1,), B, device=old.device).scatter_reduce(0, at.flatten(), b[:, None].expand(B, per).flatten(), "amin")
    refs = torch.cat((refs, refs[:1])) - gave
    frees = gone & (refs[at] == 0) & (lowest[at] == b[:, None])
    total = frees.sum()
    rank = (torch.cumsum(frees.flatten(), 0) - 1).view(B, per)
    free = torch.cat((free, free[:1])).scatter(0, torch.where(frees, count + total - 1 - rank, n).flatten(), old.flatten())[:n]
    count = count + total
    grow = (need - have).clamp(min=0)
    upto = torch.cumsum(grow, 0)
    ok = upto <= count
    fresh = ok[:, None] & (k >= have[:, None]) & (k < need[:, None])
    old = torch.where(fresh, free[(count - 1 - ((upto - grow - have)[:, None] + k)).clamp(0, n - 1)], old)
    refs = refs.scatter(0, torch.where(fresh, old, n).flatten(), 1)
    have = torch.where(ok, need, have)
    held.copy_(have)
    s["count"].copy_(count - torch.where(ok, grow, 0).sum())
    s["free"].copy_(free)
    s["refs"].copy_(refs[:n])
    table.copy_(old)
    if s["N"]:
        i = torch.arange(s["N"], device=old.device)
        b, row = i // c["rows"], i % c["rows"]
        pos = kv[b] + row
        p = pos // page
        mine = old[b, p.clamp(max=per - 1)].clamp(min=0)
        ok = (row < new[b]) & (p < have[b]) & (refs[mine] == 1)
        s["slots"].copy_(torch.where(ok, mine * page + pos % page, -1))
        s["pos"].copy_(torch.where(row < new[b], pos, -1))


def _plain_compact(s, src, dst):
    """The k-th free id below the number of live pages takes the k-th live page above it."""
    n, per, dev = s["num_pages"], s["per"], s["table"].device
    refs, ids = s["refs"].long(), torch.arange(n, device=dev)
    live = refs > 0
    count = live.sum()
    hole, mover = ~live & (ids < count), live & (ids >= count)
    m = src.numel()
    end = torch.full((m + 1,), -1, device=dev)
    frm = end.scatter(0, torch.where(mover, torch.cumsum(mover, 0) - 1, m), ids)
    to = end.scatter(0, torch.where(hole, torch.cumsum(hole, 0) - 1, m), ids)
    src.copy_(frm[:m])
    dst.copy_(to[:m])
    spare = torch.cat((ids, ids[:1]))
    spare = spare.scatter(0, torch.where(frm[:m] >= 0, frm[:m], n), to[:m])  # where each page is now
    has = torch.arange(per, device=dev) < s["held"].long()[:, None]
    s["table"].copy_(torch.where(has, spare[torch.where(has, s["table"].long(), n)], s["table"].long()))
    s["refs"].copy_(torch.zeros_like(refs).scatter_add_(0, spare[:n], refs))
    s["free"].copy_(torch.where(ids < n - count, n - 1 - ids, s["free"].long()))
    s["count"].copy_(n - count)


def _plain_copy(s, src, dst, rows):
    """The first `rows` rows of pages (None: all) to other pages, in every layer."""
    c, at = s["c"], (src >= 0).nonzero()[:, 0]
    a, b = src[at].long(), dst[at].long()
    if rows is None:
        s["kv"][:, :, b] = s["kv"][:, :, a]
        if c["f8"]:
            s["scales"][:, b] = s["scales"][:, a]
        return
    has = torch.arange(c["page"], device=at.device) < rows[at][:, None]
    s["kv"][:, :, b] = torch.where(has[:, None, :, None], s["kv"][:, :, a], s["kv"][:, :, b])
    if c["f8"]:
        s["scales"][:, b] = torch.where(has[:, None, ::32, None], s["scales"][:, a], s["scales"][:, b])


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _own_qk(s):
    import paper_2607_10661_amd as P
    c, t = s["c"], P.PTD_F32 if s["c"]["f32"] else P.PTD_BF16
    shape = P.QKShape(s["N"], c["Hq"], c["Hkv"], c["D"], c["rot"], P.PTD_ROPE_INTERLEAVED if c["inter"] else P.PTD_ROPE_HALF,
                      1 if c["norm"] else 0, t, t, s["q"].stride(0), s["k"].stride(0), s["v"].stride(0), 0, 0, EPS, THETA)
    store = P.KVStore(s["kp"].data_ptr(), s["vp"].data_ptr(), c["page"], s["num_pages"]) if c["store"] else None
    P.ptd_qk_norm_rope(s["q"], s["k"], s["v"] if c["store"] else None, s["wq"], s["wk"], s["pos"], s.get("slots"), s["q_out"],
                       s["k_out"], store, shape, None, s["status"])


def _own_logp(s):
    import paper_2607_10661_amd as P
    c = s["c"]
    P.ptd_token_logprobs(s["x"], P.PTD_F32 if c["f32"] else P.PTD_BF16, s["R"], c["V"], s["ld"], s["tokens"], s["nodes"], c["T"],
                         c["tau"], s["k"], s["logprob"], s["entropy"], s["idx"], s["val"], s["ws"], s["ws"].numel(), s["status"])


def _own_state(s, table, held):
    import paper_2607_10661_amd as P
    return P.PageState(table.data_ptr(), held.data_ptr(), s["free"].data_ptr(), s["count"].data_ptr(), s["c"]["B"], s["c"]["page"],
                       s["per"], s["num_pages"])


def _own_arrays(s):
    import paper_2607_10661_amd as P
    if "arrays" not in s:  # what a program describes once, with its caches
        c, kv = s["c"], s["kv"]
        rows = [P.PageArray(kv[i, j].data_ptr(), c["Hkv"], c["page"], 1, 128 * kv.element_size()) for i in range(c["layers"]) for j in (0, 1)]
        if c["f8"]:
            rows += [P.PageArray(x.data_ptr(), c["Hkv"], c["page"] // 32, 32, 2) for x in s["scales"]]
        s["arrays"] = (P.PageArray * len(rows))(*rows)
    return s["arrays"]


def _fork(s, table, held, frm, nxt, held2, src, dst, rows):
    if own:
        import paper_2607_10661_amd as P
        P.ptd_page_fork(_own_state(s, table, held), s["refs"], frm, s["len"], nxt, held2, src, dst, rows, s["status"])
    else:
        _plain_fork(s, table, held, frm, nxt, held2, src, dst, rows)


def _plan(s, table, held, kv, new):
    if own:
        import paper_2607_10661_amd as P
        P.ptd_page_plan_shared(_own_state(s, table, held), s["refs"], kv, new, s["N"], s["c"].get("rows", 0), s.get("start"), s["slots"],
                               s.get("pos"), s["status"])
    else:
        _plain_plan(s, table, held, kv, new)


def _compact(s, src, dst):
    if own:
        import paper_2607_10661_amd as P
        P.ptd_page_compact(_own_state(s, s["table"], s["held"]), s["refs"], src, dst, s["status"])
    else:
        _plain_compact(s, src, dst)


def _copy(s, src, dst, rows):
    if own:
        import paper_2607_10661_amd as P
        P.ptd_page_copy(_own_arrays(s), s["num_pages"], src.numel(), src, dst, rows, s["status"])
    else:
        _plain_copy(s, src, dst, rows)


def run(state):
    s, c = state, state["c"]
    if c["kind"] == "qk":
        _own_qk(s) if own else _plain_qk(s)
        return dict(q=s["q_out"], k=s["k_out"], **(dict(kp=s["kp"], vp=s["vp"]) if c["store"] else {}))
    if c["kind"] == "logp":
        _own_logp(s) if own else _plain_logp(s)
        return dict(logprob=s["logprob"], entropy=s["entropy"], **(dict(idx=s["idx"], val=s["val"]) if s["k"] else {}))
    names = ["table", "held", "refs", "free", "count"]
    if c["kind"] == "fork":
        # the samples begin (the beams go on) and get pages for their next rows; then the rows are given
        # up again, and of the samples of a prompt the first one stays
        first = [s[x + "1"] for x in ("src", "dst", "rows")]
        _fork(s, s["table"], s["held"], s["frm"], s["next"], s["held2"], *first)
        _copy(s, *first)
        _plan(s, s["next"], s["held2"], s["len"], s["new"])
        _fork(s, s["next"], s["held2"], s["back"], s["table"], s["held"], *[s[x + "2"] for x in ("src", "dst", "rows")])
        names += ["next", "held2", "slots", "pos"] + [x + i for x in ("src", "dst", "rows") for i in "12"]
    else:
        # every second sequence finishes, the others' pages are moved to the front, as many begin again
        _plan(s, s["table"], s["held"], s["half"][0], s["none"])
        _compact(s, *s["moves"][0])
        _copy(s, *s["moves"][0], None)
        _plan(s, s["table"], s["held"], s["len"], s["none"])
        _plan(s, s["table"], s["held"], s["half"][1], s["none"])
        _compact(s, *s["moves"][1])
        _copy(s, *s["moves"][1], None)
        _plan(s, s["table"], s["held"], s["len"], s["none"])
    out = {n: s[n] for n in names}
    if c["kind"] == "compact":
        out["moves"] = s["moves"]
    if c["f8"]:  # codes as the numbers they stand for, in units of their block's scale
        return dict(out, kv=s["kv"].view(torch.float8_e4m3fn), scales=s["scales"])
    return dict(out, kv=s["kv"])


# ---------------------------------------------------------------------------
# what a pass cannot do without, and its outputs in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "qk":
        N = c["B"] * c["rows"] if c["rows"] else sum(_lengths(c))
        e = 4 if c["f32"] else 2
        heads = 2 * (c["Hq"] + c["Hkv"]) + (3 * c["Hkv"] if c["store"] else 0)
        return {"bytes": N * (heads * c["D"] * e + 8), "flops": 10 * N * (c["Hq"] + c["Hkv"]) * c["D"]}
    if c["kind"] == "logp":
        r = random.Random(c["V"] * 7 + c["B"])
        n = sum(len(p) + 1 for p in _paths(c, r)) if c["path"] else c["B"]
        return {"bytes": n * c["V"] * (4 if c["f32"] else 2) + c["B"] * (c["T"] + 1) * (8 + 8 * c["k"]), "flops": 8 * n * c["V"]}
    row = c["Hkv"] * 128 * 2 * c["layers"] * (1 if c["f8"] else 2)
    page = c["page"]
    if c["kind"] == "fork":
        lens = [x for x in _lengths(c, c["groups"]) for _ in range(c["B"] // c["groups"])]
        rest = [x % page for i, x in enumerate(lens) if c["beams"] or i % (c["B"] // c["groups"])]
        # (beams: about 0.37 of them are continued by none, whose place another one's copy takes)
        moved = sum(rest) * (0.37 if c["beams"] else 1)
        return {"bytes": int(2 * moved * row + 16 * sum(-(-x // page) for x in lens) + 8 * c["B"] * c["rows"]), "flops": 0}
    need = [-(-x // page) for x in _lengths(c)]
    total, even = sum(need) + 5, sum(need[::2])
    # half of the pages of the sequences that stay lie behind the place of the last one of them
    moves = even * (total - even) / total + (sum(need) - even) * min(1.0, even / total)
    return {"bytes": int(2 * moves * row * page + 32 * sum(need)), "flops": 0}


def _exact_heads(x, w, pos, c):
    x, rot = x.double(), c["rot"]
    if c["norm"]:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS) * w.double()
    y = x.clone()
    for p in range(rot // 2):
        a, b = (2 * p, 2 * p + 1) if c["inter"] else (p, p + rot // 2)
        t = (pos.double() * math.pow(THETA, -2.0 * p / rot))[:, None]
        y[..., a] = x[..., a] * torch.cos(t) - x[..., b] * torch.sin(t)
        y[..., b] = x[..., b] * torch.cos(t) + x[..., a] * torch.sin(t)
    return y


def exact(case, seed):
    c = case
    if c["kind"] in ("fork", "compact"):
        return None
    s = prepare(case, seed)
    if c["kind"] == "qk":
        out = dict(q=_exact_heads(s["q"], s["wq"], s["pos"], c), k=_exact_heads(s["k"], s["wk"], s["pos"], c))
        if c["store"]:
            out.update(kp=torch.zeros(s["kp"].shape, dtype=torch.float64, device=DEV), vp=torch.zeros(s["vp"].shape, dtype=torch.float64, device=DEV))
            pg, row = s["slots"].long() // c["page"], s["slots"].long() % c["page"]
            out["kp"][pg, :, row], out["vp"][pg, :, row] = out["k"], s["v"].double()
        return out
    R, k, T = s["R"], s["k"], c["T"]
    out = dict(logprob=torch.zeros(R, dtype=torch.float64, device=DEV), entropy=torch.zeros(R, dtype=torch.float64, device=DEV))
    val = torch.zeros((R, k), dtype=torch.float64, device=DEV)
    tokens, nodes = s["tokens"].tolist(), s["nodes"].tolist() if c["path"] else None
    for r, t in enumerate(tokens):
        if t < 0:
            continue
        at = r if nodes is None else r - r % (T + 1) + (nodes[r // (T + 1)][r % (T + 1) - 1] + 1 if r % (T + 1) else 0)
        lp = torch.log_softmax(s["x"][at].double() / c["tau"], 0)
        out["logprob"][r] = lp[t]
        out["entropy"][r] = -torch.where(lp > -math.inf, lp * torch.exp(lp), 0.0).sum()
        if k:
            val[r] = torch.topk(lp, k).values
    return dict(out, idx=None, val=val) if k else out
