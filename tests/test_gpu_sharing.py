"""GPU checks of pages that several sequences hold: ptd_page_plan_shared, ptd_page_fork and
ptd_page_compact against a simulation with lists, ptd_page_copy against indexing, all for
equality."""
import random

import pytest
import torch

import ref64_samples as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_10661_amd as lib
    return lib


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def check_state(t, ref):
    assert t.num_held.tolist() == [len(h) for h in ref.held]
    assert t.num_free.item() == len(ref.free)
    assert t.free_pages[:len(ref.free)].tolist() == ref.free
    table = t.page_table.tolist()
    for b, h in enumerate(ref.held):
        assert table[b][:len(h)] == h
    assert t.refs.tolist() == ref.refs()


def plan(t, ref, kv, new, rows_per_seq=0, N=None):
    N = N if N is not None else (t.B * rows_per_seq if rows_per_seq else sum(new))
    st = i32([0])
    start, slots, pos = t.plan(i32(kv), i32(new), N, rows_per_seq, st)
    r_start, r_slots, r_pos, status = ref.plan(kv, new, rows_per_seq, N)
    if status == 12:
        assert st.item() in (10, 12)  # the first that was reported
    else:
        assert st.item() == status
    if not rows_per_seq:
        assert start.tolist() == r_start
    assert slots.tolist() == r_slots and pos.tolist() == r_pos
    check_state(t, ref)


def fork(t, ref, frm, length):
    st = i32([0])
    got = t.fork(i32(frm), i32(length), st)
    want = ref.fork(frm, length)
    assert st.item() == (0 if want else 12)
    if want:
        assert [x.tolist() for x in got] == [list(x) for x in want]
    else:
        assert got[0].tolist() == got[1].tolist() == [-1] * t.B and got[2].tolist() == [0] * t.B
    check_state(t, ref)
    return (*got, want is not None)


@pytest.mark.parametrize("B,page,per", [(1, 1, 12), (3, 32, 5), (8, 16, 9), (64, 16, 9), (300, 8, 4), (1100, 4, 3)])
def test_forks_and_plans_follow_the_lists(P, B, page, per):
    r = random.Random(B * page)
    num = B * per // 2 + 8
    t, ref = P.PageTables(B, page, per, num, shared=True), R.SharedPages(B, page, per, num)
    cap = page * per
    kv = [0] * B
    for s in range(10):
        # rows for some sequences, then beams: everyone continues someone, some end
        new = [r.choice([0, 0, r.randint(0, cap - k)]) if r.random() < 8 / B + 0.1 else 0 for k in kv]
        plan(t, ref, kv, new, 0 if s % 2 else max(1, max(new)))
        have = [min(k + n, len(h) * page) for k, n, h in zip(kv, new, ref.held)]
        live = [b for b in range(B) if have[b]] or [0]
        frm = [r.choice([b, r.choice(live), r.choice(live), -1]) for b in range(B)]
        length = [0 if a < 0 else r.choice([have[a], have[a], r.randint(0, have[a]), have[a] // page * page]) for a in frm]
        # (refused for want of pages: everyone stays)
        kv = length if fork(t, ref, frm, length)[3] else have
    plan(t, ref, [0] * B, [0] * B, 0, N=5)
    assert t.num_free.item() == num and (t.refs == 0).all()


@pytest.mark.parametrize("num", [8192, 8193, 32768, 32769])
def test_large_pools(P, num):
    # (the kernels' counts move from one place to another at these sizes)
    r = random.Random(num)
    B, page, per = 7, 2, 3000
    t, ref = P.PageTables(B, page, per, num, shared=True), R.SharedPages(B, page, per, num)
    kv = [0] * B
    for s in range(3):
        new, left = [0] * B, len(ref.free)
        for b in range(B):
            if kv[b] < 100:
                new[b] = r.randint(0, min(per * page - kv[b], max(0, left - 3) * page))
                left -= -(-new[b] // page) + 1
        plan(t, ref, kv, new)
        kv = [a + n for a, n in zip(kv, new)]
        frm = [r.choice([b, r.randrange(B), -1]) for b in range(B)]
        kv = [0 if a < 0 else r.randint(0, kv[a]) for a in frm]
        assert fork(t, ref, frm, kv)[3]
        st = i32([0])
        src, dst = t.compact(st)
        assert st.item() == 0 and (src.tolist(), dst.tolist()) == ref.compact()
        check_state(t, ref)


def test_samples_of_one_prompt(P):
    # 100 rows of pages of 32: three shared pages, the last one each sample's own
    t, ref = P.PageTables(5, 32, 8, 40, shared=True), R.SharedPages(5, 32, 8, 40)
    plan(t, ref, [0] * 5, [0, 0, 100, 0, 0])
    src, dst, rows, _ = fork(t, ref, [2, 2, 2, -1, 2], [100, 100, 100, 7, 96])
    assert src.tolist() == [-1, 3, 3, -1, -1] and rows.tolist() == [0, 4, 4, 0, 0]
    assert t.refs[:4].tolist() == [4, 4, 4, 1] and t.num_held.tolist() == [4, 4, 4, 0, 3]
    plan(t, ref, [100, 100, 100, 0, 96], [40, 1, 0, 0, 5], 40)
    # ends in any order; pages come back with the last holder
    plan(t, ref, [0, 100, 0, 0, 0], [0] * 5)
    assert t.refs[:3].tolist() == [1, 1, 1]
    plan(t, ref, [0] * 5, [0] * 5)
    assert t.num_free.item() == 40


def test_rows_never_go_to_shared_pages(P):
    t, ref = P.PageTables(3, 16, 6, 18, shared=True), R.SharedPages(3, 16, 6, 18)
    plan(t, ref, [0] * 3, [40, 0, 0])
    fork(t, ref, [0, 0, -1], [40, 32, 0])
    # sequence 1 is cut back into shared rows: no slot there, and the fork to itself mends it
    st = i32([0])
    _, slots, _ = t.plan(i32([40, 20, 0]), i32([2, 14, 0]), 48, 16, st)
    assert st.item() == 10
    _, want, _, _ = ref.plan([40, 20, 0], [2, 14, 0], 16, 48)
    assert slots.tolist() == want and want[16:28] == [-1] * 12 and want[28] >= 0
    src, dst, rows, _ = fork(t, ref, [0, 1, -1], [42, 20, 0])
    assert rows.tolist() == [0, 4, 0]
    plan(t, ref, [42, 20, 0], [2, 14, 0], 16)
    # many rows: the slots have a launch of their own
    t, ref = P.PageTables(2, 1024, 5, 10, shared=True), R.SharedPages(2, 1024, 5, 10)
    plan(t, ref, [0, 0], [3000, 0])
    fork(t, ref, [0, 0], [3000, 2048])
    plan(t, ref, [1500, 2048], [2000, 2500], 2500)


def test_pages_given_up_by_several_at_once(P):
    # all holders of shared pages end in one call, in rounds of sequences too
    for B, page, more in ((7, 8, 1), (200, 2, 100), (700, 4, 1), (1500, 4, 1), (300, 1, 1500)):
        t, ref = P.PageTables(B, page, 6 * more, 6 * 40 * more, shared=True), R.SharedPages(B, page, 6 * more, 6 * 40 * more)
        lens = [page * 5 * more if b < 7 else 0 for b in range(B)]
        plan(t, ref, [0] * B, lens)
        fork(t, ref, [b % 7 for b in range(B)], [page * (1 + b % 5) * (more if b < 20 else 1) for b in range(B)])
        plan(t, ref, [0 if b % 3 else page for b in range(B)], [0] * B)
        plan(t, ref, [0] * B, [page if b % 50 == 0 else 0 for b in range(B)])
        plan(t, ref, [0] * B, [0] * B)
        assert t.num_free.item() == 240 * more


@pytest.mark.parametrize("B,per,rows", [(6, 1500, 0), (6, 1500, 5000), (300, 40, 0)])
@pytest.mark.parametrize("shared", [False, True])
def test_many_pages_given_up(P, B, per, rows, shared):
    # more surplus pages than threads hold at once, of one holder or of several; with and without new rows
    r = random.Random(B)
    t, ref = P.PageTables(B, 1, per, B * per, shared=True), R.SharedPages(B, 1, per, B * per)
    kv = [r.randint(per // 2, per) for _ in range(B)]
    plan(t, ref, [0] * B, kv)
    if shared:
        frm = [b if b % 3 else 0 for b in range(B)]
        kv = [kv[a] - (0 if a == b else r.randint(0, 9)) for b, a in enumerate(frm)]
        assert fork(t, ref, frm, kv)[3]
    keep = [r.choice([0, 0, 1, r.randint(0, n)]) for n in kv]
    new = [0] * B
    new[1] = min(rows, per - keep[1])
    plan(t, ref, keep, new, N=rows)
    plan(t, ref, [0] * B, [0] * B, N=0)
    assert t.num_free.item() == B * per and (t.refs == 0).all()


def test_pages_that_are_none(P):
    # ids outside the pool and counts that are none among many surplus pages are reported, the others go back
    B, per = 4, 1200
    t = P.PageTables(B, 1, per, B * per, shared=True)
    t.plan(i32([0] * B), i32([per] * B), 0)
    t.page_table[1, 7], t.page_table[2, 8] = B * per, -5
    lost = [t.page_table[3, 9].item()]
    t.refs[lost[0]] = 0
    st = i32([0])
    before = set(range(B * per))
    t.plan(i32([0] * B), i32([0] * B), 0, dev_status=st)
    free = t.free_pages[:t.num_free.item()].tolist()
    assert st.item() == 10 and len(set(free)) == len(free) == B * per - 3 and set(free) < before and lost[0] not in free


def test_fork_refusals_change_nothing(P):
    def state():
        t = P.PageTables(4, 16, 4, 9, shared=True)
        t.plan(i32([0] * 4), i32([40, 33, 0, 20]), 93)
        return t

    t = state()
    held = [x.clone() for x in (t.page_table, t.num_held, t.refs, t.num_free, t.free_pages)]
    for frm, length, status in (([0, 1, 4, 3], [1] * 4, 13), ([0, -2, 2, 3], [0] * 4, 13), ([0, 1, 2, 3], [49, 1, 0, 1], 8),
                                ([0, 1, 2, 3], [1, -1, 0, 1], 8), ([0, 0, 0, 0], [1, 2, 2 ** 31 - 1, 1], 8),
                                ([2, 2, 2, 2], [1, 0, 0, 0], 8), ([0, 0, 0, 0], [40] * 4, 12)):
        st = i32([0])
        src, dst, rows = t.fork(i32(frm), i32(length), st)
        assert st.item() == status, (frm, length, st.item())
        assert src.tolist() == dst.tolist() == [-1] * 4 and rows.tolist() == [0] * 4
        for b, n in enumerate(held[1].tolist()):
            assert torch.equal(t.page_table[b, :n], held[0][b, :n])
        for x, y in zip((t.num_held, t.refs, t.num_free, t.free_pages), held[1:]):
            assert torch.equal(x, y)
    # a state out of range
    for field, at, value in (("num_held", 1, 5), ("num_held", 1, -1), ("num_free", 0, 10), ("num_free", 0, -1), ("page_table", (1, 0), 9),
                             ("page_table", (1, 0), -7), ("page_table", (1, 1), 2 ** 31 - 1)):
        t = state()
        getattr(t, field)[at] = value
        st = i32([0])
        src, _, _ = t.fork(i32([0, 1, -1, 3]), i32([40, 33, 0, 20]), st)
        assert st.item() == 10 and src.tolist() == [-1] * 4, (field, value)
    t = state()
    t.free_pages[0] = 99  # the page that a copy would get
    st = i32([0])
    t.fork(i32([0, 0, -1, -1]), i32([40, 40, 0, 0]), st)
    assert st.item() == 10 and t.refs.sum() == 8
    for field, value in (("num_held", 77), ("refs", 0), ("page_table", 77)):  # plans on such a state stay inside it
        t = state()
        getattr(t, field).view(-1)[1] = value
        st = i32([0])
        t.plan(i32([0] * 4), i32([0] * 4), 0, 0, st)
        assert st.item() == 10 and 0 <= t.num_free.item() <= 9


@pytest.mark.parametrize("B,page,per,num", [(1, 1, 4, 4), (4, 16, 6, 40), (40, 8, 20, 1000), (3, 4, 2, 1), (200, 4, 40, 5000)])
def test_compaction(P, B, page, per, num):
    r = random.Random(num)
    t, ref = P.PageTables(B, page, per, num, shared=True), R.SharedPages(B, page, per, num)
    kv = [0] * B
    for s in range(6):
        new, left = [0] * B, len(ref.free)
        for b in range(B):
            if kv[b] == 0 and r.random() < 0.7:
                new[b] = r.randint(0, min(per, left) * page)
                left -= -(-new[b] // page)
        plan(t, ref, kv, new)
        kv = [a + n for a, n in zip(kv, new)]
        # some end, some hold a part of others' pages, in whole pages
        frm = [r.choice([b, b, -1, r.randrange(B)]) for b in range(B)]
        kv = [kv[a] // page * page if a >= 0 else 0 for a in frm]
        fork(t, ref, frm, kv)
        st = i32([0])
        src, dst = t.compact(st)
        assert st.item() == 0 and (src.tolist(), dst.tolist()) == ref.compact()
        check_state(t, ref)
        live = num - len(ref.free)
        assert (t.refs[:live] > 0).all() and (t.refs[live:] == 0).all()


def test_compaction_of_odd_states(P):
    # lost pages come back, counts below 0 are put right, ids outside the pages stay and are reported
    t = P.PageTables(2, 4, 4, 20, shared=True)
    t.plan(i32([0, 0]), i32([16, 8]), 24)
    t.num_free.fill_(3)
    st = i32([0])
    src, dst = t.compact(st)
    assert st.item() == 0 and t.num_free.item() == 14 and t.free_pages[:14].tolist() == list(range(19, 5, -1))
    t.refs[19] = -4
    t.compact(st)
    assert st.item() == 10 and (t.refs >= 0).all()
    for field, at, value in (("page_table", (0, 1), 20), ("page_table", (0, 1), -3), ("num_held", 1, 5), ("num_held", 1, -1)):
        t = P.PageTables(2, 4, 4, 20, shared=True)
        t.plan(i32([0, 0]), i32([16, 8]), 24)
        getattr(t, field)[at] = value
        st = i32([0])
        t.compact(st)
        assert st.item() == 10 and getattr(t, field)[at] == value


@pytest.mark.parametrize("Hkv,page,D,dtype", [(1, 32, 128, torch.bfloat16), (3, 100, 64, torch.float32), (2, 7, 3, torch.uint8),
                                              (8, 64, 128, torch.uint8), (1, 1, 1, torch.uint8), (5, 64, 6, torch.bfloat16),
                                              (16, 256, 128, torch.float32)])
def test_copies(P, Hkv, page, D, dtype):
    r = random.Random(page)
    num = 23
    caches = [torch.randint(0, 250, (num, Hkv, page, D * torch.empty(0, dtype=dtype).element_size()), dtype=torch.uint8, device="cuda").view(dtype)
              for _ in range(3)]
    arrays = P.page_arrays(*caches)
    ids = r.sample(range(num), 20)
    src, dst = ids[:10], ids[10:]
    src[2] = dst[5] = -1
    dst[7] = src[7]
    src[9] = src[0]  # one page to two others
    for rows in (None, [r.choice([0, 1, page, r.randint(0, page)]) for _ in range(10)]):
        want = [x.clone() for x in caches]
        for i, (a, b) in enumerate(zip(src, dst)):
            if a >= 0 and b >= 0:
                n = page if rows is None else rows[i]
                for x, y in zip(want, caches):
                    x[b, :, :n] = y[a, :, :n]
        st = i32([0])
        P.page_copy(arrays, i32(src), i32(dst), None if rows is None else i32(rows), st)
        assert st.item() == 0
        for x, y in zip(want, caches):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_copies_of_block_scaled_pages(P):
    Hkv, page, S, num = 2, 128, 32, 9
    kv = [P.BlockKV(num, Hkv, page, S) for _ in range(3)]
    g = torch.Generator("cuda").manual_seed(0)
    for x in kv:
        k = torch.randn((2, num * page, Hkv, 128), generator=g, device="cuda").bfloat16()
        x.write(k[0], k[1], torch.arange(num * page, dtype=torch.int32, device="cuda"))
    before = [[y.clone() for y in (x.k_pages, x.v_pages, x.scales)] for x in kv]
    P.page_copy(P.page_arrays(*kv), i32([4, -1, 0]), i32([7, 2, 1]), i32([33, 5, 128]))
    for x, (k, v, s) in zip(kv, before):
        k[7, :, :33], v[7, :, :33], s[7, :, :2] = k[4, :, :33], v[4, :, :33], s[4, :, :2]
        k[1], v[1], s[1] = k[0], v[0], s[0]
        assert torch.equal(x.k_pages, k) and torch.equal(x.v_pages, v) and torch.equal(x.scales, s)


@pytest.mark.parametrize("n", [1, 63, 65, 4099, 70000])
@pytest.mark.parametrize("share", [0.0, 0.01, 1.0])
def test_copies_of_long_lists(P, n, share):
    # lists longer than the pairs that a workgroup looks up at once, most of them -1
    r = random.Random(n)
    num, Hkv, page = 600, 3, 5
    x = torch.randint(0, 250, (num, Hkv, page, 16), dtype=torch.uint8, device="cuda")
    src, dst, want = [-1] * n, [-1] * n, x.clone()
    at = r.sample(range(n), min(n, 300, int(share * n) + 1))
    for i, j in enumerate(at):
        src[j], dst[j] = r.randrange(300), 300 + i
        want[300 + i, :, :1 + j % page] = x[src[j], :, :1 + j % page]
    st = i32([0])
    P.page_copy(P.page_arrays(x), i32(src), i32(dst), i32([1 + j % page for j in range(n)]), st)
    assert st.item() == 0 and torch.equal(x, want)
    bad = src[:]
    bad[n - 1], dst[n - 1] = num, 0  # (an id outside: nothing of that pair)
    P.page_copy(P.page_arrays(x), i32(bad), i32(dst), i32([0] * n), st)
    assert st.item() == 10 and torch.equal(x, want)


@pytest.mark.parametrize("B", [1, 2, 3, 9, 15, 17, 65])
def test_forks_of_long_tables(P, B):
    # more pages than the waves of one step look at; the next tables against the old ones
    page, per = 2, 700
    r = random.Random(B)
    held = [r.choice([0, 1, 63, 64, 65, 127, 129, 600, per]) if b else per for b in range(B)]
    t = P.PageTables(B, page, per, sum(held) + 2 * B, shared=True)
    t.plan(i32([0] * B), i32([page * h for h in held]), page * sum(held))
    old = t.page_table.cpu().tolist()
    frm = [r.randrange(B) for _ in range(B)]
    ln = [r.randint(0, page * held[a]) for a in frm]
    st = i32([0])
    src, dst, rows = (v.tolist() for v in t.fork(i32(frm), i32(ln), st))
    table, refs = t.page_table.cpu().tolist(), [0] * t.num_pages
    assert st.item() == 0 and t.num_held.tolist() == [-(-x // page) for x in ln]
    for b, a in enumerate(frm):
        whole = ln[b] // page
        assert table[b][:whole] == old[a][:whole]
        if ln[b] % page:
            last = old[a][whole]
            assert (src[b], rows[b]) in ((last, ln[b] % page), (-1, 0)) and table[b][whole] == (last if src[b] < 0 else dst[b])
        for p in table[b][:-(-ln[b] // page)]:
            refs[p] += 1
    assert t.refs.tolist() == refs
    free = t.free_pages[:t.num_free.item()].tolist()
    assert sorted(free) == [p for p in range(t.num_pages) if refs[p] == 0]


def test_many_arrays_and_unaligned_ones(P):
    # more arrays than one launch takes; bases at odd addresses
    raw = torch.randint(0, 250, (200, 6 * 40 + 16), dtype=torch.uint8, device="cuda")
    arrays = [P.PageArray(raw[i].data_ptr() + i % 7, 2, 5, 2, 4) for i in range(200)]
    want = raw.clone()
    for i in range(200):
        pages = want[i, i % 7:i % 7 + 240].view(6, 2, 5, 4)
        pages[3, :, :2] = pages[1, :, :2]
    st = i32([0])
    P.ptd_page_copy(arrays, 6, 1, i32([1]), i32([3]), i32([3]), st)
    assert torch.equal(raw, want) and st.item() == 0


def test_refused_copies(P):
    x = torch.randint(0, 250, (5, 2, 8, 16), dtype=torch.uint8, device="cuda")
    keep, arrays = x.clone(), P.page_arrays(x[:4])
    for src, dst, rows, status in ((4, 0, None, 10), (0, 4, None, 10), (-2, 0, None, 10), (0, 2 ** 31 - 1, None, 10), (0, 1, 9, 13), (0, 1, -1, 13)):
        st = i32([0])
        P.page_copy(arrays, i32([src]), i32([dst]), None if rows is None else i32([rows]), st)
        assert st.item() == status and torch.equal(x, keep)


def test_pages_past_32_bits(P):
    # a cache of more than 2^32 bytes: its last pages
    n = (1 << 32) // (8 * 64 * 256) + 40
    x = torch.zeros((n, 8, 64, 256), dtype=torch.uint8, device="cuda")
    x[n - 1] = 9
    x[3] = 5
    P.page_copy(P.page_arrays(x), i32([n - 1, 3]), i32([1, n - 2]), i32([64, 10]))
    assert (x[1] == 9).all() and (x[n - 2, :, :10] == 5).all() and (x[n - 2, :, 10:] == 0).all()


def test_in_a_graph(P):
    B, page, per, num = 6, 16, 8, 60
    t, ref = P.PageTables(B, page, per, num, shared=True), R.SharedPages(B, page, per, num)
    cache = torch.randint(0, 250, (num, 2, page, 16), dtype=torch.uint8, device="cuda")
    arrays = P.page_arrays(cache)
    plan(t, ref, [0] * B, [50, 0, 0, 20, 0, 0])
    frm, ln, kv, new = (i32([0] * B) for _ in range(4))
    nxt, held = torch.full_like(t.page_table, -1), torch.zeros_like(t.num_held)
    src, dst, rows, slots, st = i32([0] * B), i32([0] * B), i32([0] * B), i32([0] * (B * 4)), i32([0])
    ms, md = i32([0] * (num // 2)), i32([0] * (num // 2))
    state2 = P.PageState(nxt.data_ptr(), held.data_ptr(), t.free_pages.data_ptr(), t.num_free.data_ptr(), B, page, per, num)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.ptd_page_fork(t.state(), t.refs, frm, ln, nxt, held, src, dst, rows, st)
        P.ptd_page_copy(arrays, num, B, src, dst, rows, st)
        P.ptd_page_plan_shared(state2, t.refs, kv, new, B * 4, 4, None, slots, None, st)
        P.ptd_page_compact(state2, t.refs, ms, md, st)
        P.ptd_page_copy(arrays, num, num // 2, ms, md, None, st)
        t.page_table.copy_(nxt)
        t.num_held.copy_(held)
    kvs = [50, 0, 0, 20, 0, 0]
    for a, more in (([0, 0, 3, 3, 0, -1], 4), ([0, 1, 2, 3, 4, 2], 3), ([4, 4, 4, 4, 4, 4], 1), ([1, 1, -1, 0, 5, 2], 2)):
        n = [kvs[x] if x >= 0 else 0 for x in a]
        want = cache.clone()
        c = ref.fork(a, n)
        for s_, d_, r_ in zip(*c):
            if s_ >= 0:
                want[d_, :, :r_] = want[s_, :, :r_]
        _, w_slots, _, _ = ref.plan(n, [more] * B, 4, B * 4)
        m = ref.compact()
        moved = want.clone()
        for s_, d_ in zip(*m):
            if s_ >= 0:
                moved[d_] = want[s_]
        frm.copy_(i32(a)), ln.copy_(i32(n)), kv.copy_(i32(n)), new.copy_(i32([more] * B))
        g.replay()
        torch.cuda.synchronize()
        assert slots.tolist() == w_slots and st.item() == 0
        check_state(t, ref)
        assert torch.equal(cache, moved)
        kvs = [x + more for x in n]


def test_plans_without_sharing_are_those_of_ptd_page_plan(P):
    r = random.Random(5)
    a, b = P.PageTables(20, 16, 9, 170), P.PageTables(20, 16, 9, 170, shared=True)
    kv = [0] * 20
    for _ in range(8):
        new = [r.randint(0, 144 - k) if r.random() < 0.5 else 0 for k in kv]
        x, y = a.plan(i32(kv), i32(new), sum(new)), b.plan(i32(kv), i32(new), sum(new))
        for u, v in zip(x, y):
            assert torch.equal(u, v)
        n = a.num_free.item()
        assert torch.equal(a.free_pages[:n], b.free_pages[:n]) and n == b.num_free.item()
        kv = [0 if r.random() < 0.3 else k + r.randint(0, m) for k, m in zip(kv, new)]


def test_helpers_refuse(P):
    t = P.PageTables(2, 16, 4, 8)
    with pytest.raises(ValueError):
        t.fork(i32([0, 0]), i32([0, 0]))
    with pytest.raises(ValueError):
        t.compact()
    t = P.PageTables(2, 16, 4, 8, shared=True)
    with pytest.raises(ValueError):
        t.fork(i32([0]), i32([0, 0]))
    with pytest.raises(ValueError):
        t.fork(i32([0, 0]).long(), i32([0, 0]))
    x = torch.zeros((4, 2, 8, 16), device="cuda")
    with pytest.raises(ValueError):
        P.page_arrays(x, x[:3])
    with pytest.raises(ValueError):
        P.page_arrays(x[:, :, ::2])
    with pytest.raises(ValueError):
        P.page_copy(P.page_arrays(x), i32([0]), i32([0, 1]))


def test_tables_work_with_the_attention(P):
    # two samples over shared 8-bit pages attend as two sequences with pages of their own
    Hq, Hkv, page, S, B, per = 4, 2, 64, 32, 3, 6
    t, st = P.PageTables(B, page, per, B * per, shared=True), i32([0])
    kv = P.BlockKV(B * per, Hkv, page, S)
    g = torch.Generator("cuda").manual_seed(7)
    x = torch.randn((150, Hq + 2 * Hkv, 128), generator=g, device="cuda").bfloat16()
    _, slots, pos = t.plan(i32([0, 0, 0]), i32([150, 0, 0]), 150, dev_status=st)
    kv.write(x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], slots, dev_status=st)
    c = t.fork(i32([0, 0, 0]), i32([150, 150, 150]), st)
    P.page_copy(P.page_arrays(kv), *c, dev_status=st)
    y = torch.randn((B, 4, Hq + 2 * Hkv, 128), generator=g, device="cuda").bfloat16()
    lens = i32([150] * 3)
    _, slots, _ = t.plan(lens, i32([4] * 3), 12, 4, st)
    f = y.flatten(0, 1)
    kv.write(f[:, Hq:Hq + Hkv], f[:, Hq + Hkv:], slots, dev_status=st)
    parent = i32([[-1, 0, 0, 2]] * 3)
    q = y[:, :, :Hq].contiguous()
    out = kv.tree_attention(q, t.page_table, lens, parent, out_dtype=torch.float32, dev_status=st)
    for b in range(B):
        other = P.BlockKV(per, Hkv, page, S)
        k, v = (torch.cat((x[:, a:a + Hkv], y[b, :, a:a + Hkv])) for a in (Hq, Hq + Hkv))
        other.write(k[:150], v[:150], torch.arange(150, dtype=torch.int32, device="cuda"))
        other.write(k[150:], v[150:], torch.arange(150, 154, dtype=torch.int32, device="cuda"))
        alone = other.tree_attention(q[b:b + 1], i32([list(range(per))]), lens[:1], parent[:1], out_dtype=torch.float32)
        # the same rows, weights and tiles, in a batch of another size: sums in another order
        ids = t.page_table[b, :3].long()
        assert torch.equal(kv.k_pages[ids].transpose(1, 2).reshape(-1, Hkv, 128)[:154], other.k_pages[:3].transpose(1, 2).reshape(-1, Hkv, 128)[:154])
        assert (out[b] - alone[0]).abs().max() <= 2.0 ** -7 * 4 and st.item() == 0
