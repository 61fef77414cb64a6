"""GPU check of serving several samples of one prompt as a whole: prompts are normed, turned, attended to and
written into 8-bit pages; each prompt becomes several samples that share its pages; steps of draft trees
follow (norm and rotation of the tree rows, pages of their own, attention, verification, log
probabilities of the emitted tokens, commit); the likelier samples replace the others; pages are moved
together.  Outputs are compared with plain 64-bit implementations on each sample's own rows."""
import random

import numpy as np
import pytest
import torch

import ref64
import ref64_samples as R
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


@pytest.mark.parametrize("page,S,layers", [(64, 32, 2), (128, 128, 1)])
def test_samples_of_prompts(P, page, S, layers):
    B, prompts, T, Hq, Hkv, V, per, steps = 6, 2, 16, 4, 2, 700, 8, 4
    r, rng = random.Random(page), np.random.default_rng(page)
    g = torch.Generator("cuda").manual_seed(page)
    tables, st = P.PageTables(B, page, per, B * per, shared=True), i32([0])
    kv = [P.BlockKV(B * per, Hkv, page, S) for _ in range(layers)]
    arrays = P.page_arrays(*kv)
    wq, wk = ((1 + 0.1 * torch.randn(128, generator=g, device="cuda")).bfloat16() for _ in range(2))
    true = [[[torch.zeros((0, Hkv, 128)) for _ in range(2)] for _ in range(layers)] for _ in range(B)]  # rows as computed

    def normed(n, pos):
        """Queries and keys of n rows, normed and turned in place of a projection, and values."""
        x = torch.randn((n, Hq + 2 * Hkv, 128), generator=g, device="cuda").bfloat16()
        q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        f = [10000.0 ** (-2.0 * p / 128) for p in range(64)]
        want = [R.heads(y, w, pos, f, 128, False, 1e-6) for y, w in ((q, wq), (k, wk))]
        P.qk_norm_rope(q, k, pos, wq, wk, q_out=q, k_out=k, dev_status=st)
        live = pos >= 0
        for got, (ref, mag) in zip((q, k), want):
            assert ((got.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -19 * mag)[live].all()
        return q, k, v

    def check_rows():
        for b in range(B):
            for l in range(layers):
                if lens[b]:
                    for got, want in zip(cached(kv[l], tables, b, lens[b]), true[b][l]):
                        x, y = want.double().transpose(0, 1), got.double().cpu()
                        # half a step of a code, twice the least step of the block's scale (a row
                        # can have been coded under a larger one before)
                        assert ((x - y).abs() <= 2.0 ** -4 * x.abs() + 2.0 ** -9 * 2 * x.abs().amax() / 224).all()

    # the prompts, in the first sequence of each group
    group = B // prompts
    lens = [r.randint(60, 200) if b % group == 0 else 0 for b in range(B)]
    start, slots, pos = tables.plan(i32([0] * B), i32(lens), sum(lens), dev_status=st)
    at = start.tolist()
    for l in range(layers):
        q, k, v = normed(sum(lens), pos)
        out = P.prompt_attention(q, k, v, start, out_dtype=torch.float32, dev_status=st)
        ref, mag, _ = ref64.causal(q, k, v, at, 128 ** -0.5)
        assert ((out.double() - ref).abs() <= (2.0 ** -8 + 2.0 ** -11) * mag + 2.0 ** -8 * ref.abs()).all()
        kv[l].write(k, v, slots, dev_status=st)
        for b in range(B):
            true[b][l] = [x[at[b]:at[b + 1]].cpu() for x in (k, v)]
    check_rows()

    def go_on(frm, length):
        nonlocal lens, true
        c = tables.fork(i32(frm), i32(length), st)
        P.page_copy(arrays, *c, dev_status=st)
        lens = list(length)
        true = [[[x[:n] for x in true[max(a, 0)][l]] for l in range(layers)] for a, n in zip(frm, length)]

    go_on([b // group * group for b in range(B)], [lens[b // group * group] for b in range(B)])
    check_rows()
    assert (tables.refs > 1).any()
    score = [0.0] * B
    for n in range(steps):
        parent = np.stack([W.tree_uniform(rng, T)[0] for _ in range(B)])
        tokens = np.stack([W.sibling_distinct_tokens(rng, parent[b], V) for b in range(B)])
        pos = P.tree_rope(None, torch.zeros((B, 1, per * page, 128), dtype=torch.bfloat16, device="cuda"), i32(lens), i32(parent), dev_status=st)
        _, slots, _ = tables.plan(i32(lens), i32([T] * B), B * T, T, st)
        assert (slots >= 0).all()
        rows = []
        for l in range(layers):
            q, k, v = normed(B * T, pos.view(-1))
            rows.append((k.cpu(), v.cpu()))
            kv[l].write(k, v, slots, dev_status=st)
            out = kv[l].tree_attention(q.reshape(B, T, Hq, 128).contiguous(), tables.page_table, i32(lens), i32(parent),
                                       out_dtype=torch.float32, dev_status=st)
            for b in range(B):
                kc, vc = cached(kv[l], tables, b, lens[b] + T)
                ref, mag = ref64.tree(q[b * T:(b + 1) * T], kc, vc, lens[b], parent[b], 128 ** -0.5, T)
                assert ((out[b].double() - ref).abs() <= (2.0 ** -8 + 2.0 ** -11) * mag + 2.0 ** -8 * ref.abs()).all()
            last = k, v
        logits = torch.randn((B, T + 1, V), generator=g, device="cuda").mul_(2).bfloat16()
        for b in range(B):  # a planted path is accepted
            a, path = r.randrange(-1, T), []
            while a >= 0:
                path.append(a)
                a = int(parent[b, a])
            prev = 0
            for a in path[::-1]:
                logits[b, prev, tokens[b, a]] = 14.0
                prev = a + 1
        am, _, _ = P.topk_argmax(logits, 1)
        al, an, ot = P.verify(am.view(B, T + 1), i32(tokens), i32(parent), dev_status=st)
        lp, ent, idx, val = P.token_logprobs(logits, ot.view(-1), 2, nodes=an, dev_status=st)
        lp = lp.view(B, T + 1)
        for b, m in enumerate(al.tolist()):
            at = [0] + [x + 1 for x in an[b, :m].tolist()]
            for j in range(T + 1):
                i = b * (T + 1) + j
                if j > m:
                    assert lp[b, j] == 0 and ent[i] == 0 and (idx[i] == -1).all()
                    continue
                w_lp, w_ent, order, _, e_lp, e_ent = R.logprobs(logits[b, at[j]].cpu(), 1.0, ot[b, j].item(), 2)
                assert abs(lp[b, j].item() - w_lp) <= e_lp + 2.0 ** -24 * abs(w_lp) and abs(ent[i].item() - w_ent) <= e_ent
                assert idx[i].tolist() == order and val[i, 0] == lp[b, j]  # greedy: the likeliest
            score[b] += lp[b].sum().item()
        _, slots, _ = tables.plan(i32(lens), al, B * T, T, st)
        for l in range(layers):
            k, v = rows[l]
            kv[l].write(k.cuda(), v.cuda(), slots, src=an, rows_per_seq=T, dev_status=st)
            for b, m in enumerate(al.tolist()):
                src = [b * T + x for x in an[b, :m].tolist()]
                true[b][l] = [torch.cat((x, y[src])) for x, y in zip(true[b][l], rows[l])]
        lens = [a + m for a, m in zip(lens, al.tolist())]
        check_rows()
        # the best of each group goes on in all of its places but one, which ends
        frm = []
        for p in range(prompts):
            mine = sorted(range(p * group, (p + 1) * group), key=lambda b: -score[b])
            frm += [mine[0]] * (group - 1) + [mine[1] if n % 2 else -1]
        score = [0.0 if a < 0 else score[a] for a in frm]
        go_on(frm, [0 if a < 0 else lens[a] for a in frm])
        check_rows()
        if n % 2 == 0:
            P.page_copy(arrays, *tables.compact(st), dev_status=st)
            live = tables.num_free.item()
            assert (tables.refs[B * per - live:] == 0).all() and (tables.refs[:B * per - live] > 0).all()
            check_rows()
    tables.plan(i32([0] * B), i32([0] * B), 0, 0, st)
    assert tables.num_free.item() == B * per and (tables.refs == 0).all() and st.item() == 0
