"""GPU check of the serving path as a whole: prompts are attended to and written into
8-bit pages that ptd_page_plan hands out, then steps of a draft tree follow (tree rows
written, attended to, verified, the accepted ones committed), sequences finish and
new prompts take their pages.  Every output is compared with a plain 64-bit implementation
on the rows that the cache stands for, the rows with those written."""
import random

import numpy as np
import pytest
import torch

import ref64
import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_10661_amd as lib
    return lib


def i32(x):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32).cuda()


def cached(kv, tables, b, n):
    """Rows 0 .. n - 1 of sequence b as bf16 [Hkv][n][128] (exact), for keys and values."""
    ids = tables.page_table[b, :-(-n // kv.page_size)].long()
    got = []
    for kind, x in enumerate((kv.k_pages, kv.v_pages)):
        y = x[ids].view(torch.float8_e4m3fn).double().unflatten(2, (-1, kv.scale_rows))
        y = (y * torch.exp2(kv.scales[ids][..., kind].double() - 127)[..., None, None]).flatten(2, 3)
        got.append(y.transpose(0, 1).reshape(kv.Hkv, -1, 128)[:, :n].bfloat16())
    return got


@pytest.mark.parametrize("Hq,Hkv,page,S", [(8, 2, 64, 32), (4, 4, 128, 128)])
def test_prompts_steps_and_turnover(P, Hq, Hkv, page, S):
    B, T, per, steps = 4, 24, 8, 5
    r, rng = random.Random(Hq), np.random.default_rng(Hq)
    g = torch.Generator("cuda").manual_seed(Hq)
    tables = P.PageTables(B, page, per, B * per)
    kv = P.BlockKV(B * per, Hkv, page, S)
    st = i32([0])
    true = [[torch.zeros((0, Hkv, 128)), torch.zeros((0, Hkv, 128))] for _ in range(B)]  # rows as computed
    lens = [0] * B

    def rows(n):
        x = torch.randn((n, Hq + 2 * Hkv, 128), generator=g, device="cuda").bfloat16()
        return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]

    def check_rows():
        for b in range(B):
            if lens[b]:
                for got, want in zip(cached(kv, tables, b, lens[b]), true[b]):
                    x, y = want.double().transpose(0, 1), got.double().cpu()
                    # half a step of a code, twice the least step of the block's scale (a row
                    # can have been coded under a larger one before)
                    top = x.abs().amax()
                    assert ((x - y).abs() <= 2.0 ** -4 * x.abs() + 2.0 ** -9 * 2 * top / 224).all()

    def admit(prompts):
        """prompts[b] rows for the sequences that start anew, none for the others."""
        q, k, v = rows(sum(prompts))
        start, slots, pos = tables.plan(i32(lens), i32(prompts), sum(prompts), dev_status=st)
        out = P.prompt_attention(q, k, v, start, dev_status=st, out_dtype=torch.float32)
        kv.write(k, v, slots, dev_status=st)
        s = start.tolist()
        ref, mag, _ = ref64.causal(q, k, v, s, 128 ** -0.5)
        assert ((out.double() - ref).abs() <= (2.0 ** -8 + 2.0 ** -11) * mag + 2.0 ** -8 * ref.abs()).all()
        for b in range(B):
            if prompts[b]:
                assert pos[s[b]:s[b + 1]].tolist() == list(range(prompts[b]))
                true[b] = [x[s[b]:s[b + 1]].cpu() for x in (k, v)]
                lens[b] = prompts[b]

    admit([100, 1, 257, 64])
    check_rows()
    for n in range(steps):
        parent = np.stack([W.tree_uniform(rng, T)[0] for _ in range(B)])
        tokens = np.stack([W.sibling_distinct_tokens(rng, parent[b], 500) for b in range(B)])
        q, k, v = rows(B * T)
        _, slots, _ = tables.plan(i32(lens), i32([T] * B), B * T, T, st)
        kv.write(k, v, slots, dev_status=st)
        out = kv.tree_attention(q.reshape(B, T, Hq, 128).contiguous(), tables.page_table, i32(lens), i32(parent),
                                out_dtype=torch.float32, dev_status=st)
        for b in range(B):
            kc, vc = cached(kv, tables, b, lens[b] + T)
            ref, mag = ref64.tree(q[b * T:(b + 1) * T], kc, vc, lens[b], parent[b], 128 ** -0.5, T)
            # (the weights are rounded to bf16 above and below the line)
            assert ((out[b].double() - ref).abs() <= (2.0 ** -8 + 2.0 ** -11) * mag + 2.0 ** -8 * ref.abs()).all()
        # a planted path is accepted
        argmax = np.full((B, T + 1), 777, np.int32)
        for b in range(B):
            a, path = r.randrange(-1, T), []
            while a >= 0:
                path.append(a)
                a = int(parent[b, a])
            prev = 0
            for a in path[::-1]:
                argmax[b, prev] = tokens[b, a]
                prev = a + 1
        al, an, _ = P.verify(i32(argmax), i32(tokens), i32(parent), dev_status=st)
        _, slots, pos = tables.plan(i32(lens), al, B * T, T, st)
        kv.write(k, v, slots, src=an, rows_per_seq=T, dev_status=st)
        for b, m in enumerate(al.tolist()):
            src = [b * T + x for x in an[b, :m].tolist()]
            true[b] = [torch.cat((x, y[src].cpu())) for x, y in zip(true[b], (k, v))]
            assert pos[b * T:b * T + m].tolist() == list(range(lens[b], lens[b] + m))
            lens[b] += m
        check_rows()
        assert tables.num_held.tolist() == [-(-x // page) for x in lens]
        if n == 2:  # two sequences finish, new prompts take their pages
            lens[0] = lens[2] = 0
            tables.plan(i32(lens), i32([0] * B), 0, 1 * 0, st)
            admit([33, 0, 130, 0])
            check_rows()
    tables.plan(i32([0] * B), i32([0] * B), 0, 0, st)
    assert tables.num_free.item() == B * per and st.item() == 0


def test_what_a_rejected_row_costs(P):
    # 20 committed rows, then a tree with one node 2^12 times as large as the others, which is
    # rejected: its scale is gone with the commit, the places lost under it are not
    S, T, Hkv = 32, 8, 2
    tables, kv, st = P.PageTables(1, 64, 2, 2), P.BlockKV(2, Hkv, 64, S), i32([0])
    g = torch.Generator("cuda").manual_seed(3)
    k, v = (torch.randn((20, Hkv, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
    kv.write(k, v, tables.plan(i32([0]), i32([20]), 20, dev_status=st)[1], dev_status=st)
    page = tables.page_table[0, 0].item()
    first = torch.exp2(kv.scales[page, :, 0].double() - 127)  # [Hkv][2]
    tk, tv = (torch.randn((T, Hkv, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
    tk[5] *= 4096
    tv[5] *= 4096
    kv.write(tk, tv, tables.plan(i32([20]), i32([T]), T, T, st)[1], dev_status=st)
    large = torch.exp2(kv.scales[page, :, 0].double() - 127)
    assert (large >= 1024 * first).all()
    _, slots, _ = tables.plan(i32([20]), i32([2]), T, T, st)
    kv.write(tk, tv, slots, src=i32([0, 3] + [-1] * 6), rows_per_seq=T, dev_status=st)
    assert (torch.exp2(kv.scales[page, :, 0].double() - 127) < large / 256).all() and st.item() == 0
    for kind, (x, got) in enumerate(zip((k, v), cached(kv, tables, 0, 20))):
        x, off = x.double().transpose(0, 1), (x.double().transpose(0, 1) - got.double()).abs()
        step0, step1 = (s[:, kind, None, None] for s in (first, large))
        assert (off <= torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -10 * step0) + 2.0 ** -10 * step1).all()
    for x, got in zip((tk, tv), cached(kv, tables, 0, 22)):
        x, now = x[[0, 3]].double().transpose(0, 1), torch.exp2(kv.scales[page, :, 0].double() - 127).amax()
        assert ((x - got[:, 20:].double()).abs() <= torch.clamp(2.0 ** -4 * x.abs(), min=2.0 ** -10 * now)).all()


@pytest.mark.parametrize("page,S", [(32, 32), (64, 32), (128, 128)])
def test_last_blocks_written_anew_hold_no_trace_of_rejected_rows(P, page, S):
    # the rows of a sequence's last block are kept as they were, and a commit writes that
    # block from its first row: the cache is that of one write of all rows
    B, T, Hkv, per, steps = 4, 16, 2, 8, 12
    R = S + T
    r, g = random.Random(page + S), torch.Generator("cuda").manual_seed(S)
    tables, kv, st = P.PageTables(B, page, per, B * per), P.BlockKV(B * per, Hkv, page, S), i32([0])

    def rows(n):
        return torch.randn((2, n, Hkv, 128), generator=g, device="cuda").bfloat16()

    lens = [5, S, 0, S + 7]
    x = rows(sum(lens))
    kv.write(*x, tables.plan(i32([0] * B), i32(lens), sum(lens), dev_status=st)[1], dev_status=st)
    true = [x[:, sum(lens[:b]):sum(lens[:b + 1])] for b in range(B)]
    for n in range(steps):
        x = rows(B * T).unflatten(1, (B, T))
        wild = [r.sample(range(T), 3) for _ in range(B)]
        for b in range(B):
            x[:, b, wild[b]] *= 2.0 ** 14
        _, slots, _ = tables.plan(i32(lens), i32([T] * B), B * T, T, st)
        kv.write(*x.flatten(1, 2), slots, dev_status=st)
        good = [[t for t in range(T) if t not in wild[b]] for b in range(B)]
        acc = [sorted(r.sample(good[b], r.randint(0, 6))) for b in range(B)]
        off = [a % S for a in lens]
        both = torch.zeros((2, B, R, Hkv, 128), device="cuda", dtype=torch.bfloat16)
        both[:, :, S:] = x
        for b in range(B):
            both[:, b, :off[b]] = true[b][:, lens[b] - off[b]:]
        src = [list(range(off[b])) + [S + a for a in acc[b]] for b in range(B)]
        _, slots, _ = tables.plan(i32([a - o for a, o in zip(lens, off)]), i32([len(y) for y in src]), B * R, R, st)
        kv.write(*both.flatten(1, 2), slots, src=i32([y + [-1] * (R - len(y)) for y in src]), rows_per_seq=R, dev_status=st)
        true = [torch.cat((true[b], x[:, b, acc[b]]), 1) for b in range(B)]
        lens = [a + len(c) for a, c in zip(lens, acc)]
    other = P.BlockKV(B * per, Hkv, page, S)
    tables.plan(i32(lens), i32([0] * B), 0, dev_status=st)
    slots = torch.cat([(tables.page_table[b, :, None] * page + torch.arange(page, device="cuda")).flatten()[:lens[b]]
                       for b in range(B)]).int().contiguous()
    other.write(*torch.cat(true, 1), slots, dev_status=st)
    assert st.item() == 0
    at = slots.long()
    for a, b in ((kv.k_pages, other.k_pages), (kv.v_pages, other.v_pages)):
        assert torch.equal(a[at // page, :, at % page], b[at // page, :, at % page])
    assert torch.equal(kv.scales[at // page, :, at % page // S], other.scales[at // page, :, at % page // S])
