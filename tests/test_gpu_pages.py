"""GPU checks of page tables and slot maps (ptd_page_init, ptd_page_plan) against a
plain simulation with lists, and of rows written into 8-bit pages with block scales
(ptd_kv_write_fp8blk) against the format's definition in 64 bits.  Everything is
compared for equality: a power-of-two scale and a rounding to nearest even are exact."""
import random

import numpy as np
import pytest
import torch

import ref64

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


def step(P, t, ref, kv, new, rows_per_seq, status=0, N=None):
    N = N if N is not None else (t.B * rows_per_seq if rows_per_seq else sum(new))
    st = i32([0])
    start, slots, pos = t.plan(i32(kv), i32(new), N, rows_per_seq, st)
    assert st.item() == status, st.item()
    r_start, r_slots, r_pos = ref.plan(kv, new, rows_per_seq, N)
    if not rows_per_seq:
        assert start.tolist() == r_start
    assert slots.tolist() == r_slots and pos.tolist() == r_pos
    check_state(t, ref)


@pytest.mark.parametrize("B,page,per", [(1, 1, 40), (3, 32, 5), (16, 64, 20), (64, 16, 9), (513, 8, 4), (1100, 4, 3)])
@pytest.mark.parametrize("packed", [False, True])
def test_plans_follow_the_lists(P, B, page, per, packed):
    r = random.Random(B * page + packed)
    num = B * per + 3
    t, ref = P.PageTables(B, page, per, num), ref64.Pages(B, page, per, num)
    check_state(t, ref)
    kv = [0] * B
    for s in range(6):
        cap = page * per
        new = [r.choice([0, 1, r.randint(0, cap - k)]) if k < cap else 0 for k in kv]
        step(P, t, ref, kv, new, 0 if packed else max(1, max(new)))
        # some rows are kept, some sequences finish
        kv = [0 if r.random() < 0.2 else k + r.randint(0, n) for k, n in zip(kv, new)]
    step(P, t, ref, [0] * B, [0] * B, 0, N=5)
    assert t.num_free.item() == num


def test_many_rows(P):
    # more rows than the planning workgroup writes: the slots have a launch of their own
    B, page, per = 9, 64, 80
    t, ref = P.PageTables(B, page, per, B * per), ref64.Pages(B, page, per, B * per)
    step(P, t, ref, [0] * B, [5120, 0, 1, 4000, 64, 63, 65, 0, 2500], 0)
    step(P, t, ref, [0] * B, [5120, 0, 1, 4000, 64, 63, 65, 0, 2500], 0, N=20000)
    step(P, t, ref, [100, 3, 0, 0, 64, 1, 2, 3, 2000], [1500] * B, 1500)
    B = 700  # more sequences than threads
    t, ref = P.PageTables(B, 4, 20, B * 20), ref64.Pages(B, 4, 20, B * 20)
    step(P, t, ref, [i % 7 for i in range(B)], [i % 50 for i in range(B)], 0)
    step(P, t, ref, [i % 5 for i in range(B)], [i % 49 for i in range(B)], 48 + 1)


def test_trim_undoes_growth(P):
    t = P.PageTables(4, 32, 8, 40)
    t.plan(i32([40, 0, 100, 7]), i32([0, 0, 0, 0]), 0, 1 * 0)
    before = [x.clone() for x in (t.num_held, t.free_pages, t.num_free)]
    t.plan(i32([40, 0, 100, 7]), i32([64, 64, 64, 64]), 256, 64)
    assert t.num_free.item() < before[2].item()
    t.plan(i32([40, 0, 100, 7]), i32([0] * 4), 256, 64)
    assert torch.equal(t.num_held, before[0]) and torch.equal(t.num_free, before[2])
    n = before[2].item()
    assert torch.equal(t.free_pages[:n], before[1][:n])


@pytest.mark.parametrize("packed", [False, True])
def test_too_few_pages(P, packed):
    # the third sequence does not fit; the fourth would, but comes after it
    t, ref = P.PageTables(5, 16, 10, 12), ref64.Pages(5, 16, 10, 12)
    step(P, t, ref, [0] * 5, [32, 64, 150, 16, 0], 0 if packed else 150, status=12)
    assert t.num_held.tolist() == [2, 4, 0, 0, 0] and t.num_free.item() == 6
    # pages given back in the same call are there for the others
    step(P, t, ref, [0] * 5, [0, 0, 150, 16, 0], 0 if packed else 150)
    assert t.num_held.tolist() == [0, 0, 10, 1, 0]
    # refused across rounds of sequences
    B = 1200
    t, ref = P.PageTables(B, 4, 4, 600), ref64.Pages(B, 4, 4, 600)
    step(P, t, ref, [0] * B, [(i % 3) * 2 for i in range(B)], 0 if packed else 4, status=12)


def test_refused_lengths(P):
    for kv, new in (([-1, 5], [3, 3]), ([5, 5], [-1, 3]), ([60, 5], [5, 3]), ([2 ** 31 - 1, 5], [2 ** 31 - 1, 3])):
        t = P.PageTables(2, 16, 4, 20)
        st = i32([0])
        start, slots, pos = t.plan(i32(kv), i32(new), 6, 0, st)
        assert st.item() == 8
        # the other sequence is served, in the refused one's place
        assert start.tolist() == [0, 0, 3] and t.num_held.tolist() == [0, 1]
        assert slots.tolist()[:3] == [5, 6, 7] and slots.tolist()[3:] == [-1] * 3
        assert pos.tolist() == [5, 6, 7, -1, -1, -1]


def test_more_rows_than_room(P):
    t = P.PageTables(2, 16, 4, 20)
    st = i32([0])
    start, slots, _ = t.plan(i32([0, 0]), i32([10, 10]), 15, 0, st)
    assert st.item() == 13 and start.tolist() == [0, 10, 20]
    assert slots.tolist() == list(range(10)) + list(range(16, 21))
    st = i32([0])
    _, slots, _ = t.plan(i32([0, 0]), i32([10, 3]), 16, 8, st)
    assert st.item() == 13
    assert slots.tolist() == list(range(8)) + [16, 17, 18] + [-1] * 5


def test_state_out_of_range_is_reported(P):
    for field, value in (("num_held", [-1, 0]), ("num_held", [5, 0]), ("num_free", [21]), ("num_free", [-2])):
        t = P.PageTables(2, 16, 4, 20)
        getattr(t, field).copy_(i32(value))
        st = i32([0])
        t.plan(i32([0, 0]), i32([10, 3]), 13, 0, st)
        assert st.item() == 10, (field, value)
    # an id outside the pages: no slot
    t = P.PageTables(1, 16, 4, 20)
    t.plan(i32([0]), i32([40]), 0, 0)
    t.page_table[0, 1] = 20
    st = i32([0])
    _, slots, _ = t.plan(i32([0]), i32([40]), 40, 0, st)
    assert st.item() == 10
    assert slots.tolist() == list(range(16)) + [-1] * 16 + list(range(32, 40))


def test_plan_in_a_graph(P):
    t, ref = P.PageTables(3, 16, 6, 18), ref64.Pages(3, 16, 6, 18)
    kv, new = i32([0, 0, 0]), i32([0, 0, 0])
    slots, pos, start = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (96, 96, 4))
    st = i32([0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.ptd_page_plan(t.state(), kv, new, 96, 0, start, slots, pos, st)
    for a, b in (([0, 0, 0], [20, 3, 40]), ([20, 3, 40], [10, 0, 7]), ([5, 0, 47], [0, 90, 1]), ([0] * 3, [0] * 3)):
        kv.copy_(i32(a))
        new.copy_(i32(b))
        g.replay()
        torch.cuda.synchronize()
        want = ref.plan(a, b, 0, 96)
        assert (start.tolist(), slots.tolist(), pos.tolist()) == want and st.item() == 0
        check_state(t, ref)


# ---------------------------------------------------------------------------
# rows into pages
# ---------------------------------------------------------------------------
def values(codes):
    return codes.view(torch.float8_e4m3fn).double().cpu().numpy()


class Blocks:
    """The cache's content as numbers: (page, block) -> (codes' values, exponent) for
    each head and kind."""

    def __init__(self, kv):
        self.S, self.blocks = kv.scale_rows, kv.page_size // kv.scale_rows
        self.c = [values(x).reshape(kv.num_pages, kv.Hkv, self.blocks, self.S, 128) for x in (kv.k_pages, kv.v_pages)]
        self.e = kv.scales.cpu().numpy().astype(int) - 127
        self.Hkv = kv.Hkv

    def write(self, rows, slots):
        """rows: (k, v) float64 [n][Hkv][128] in the order of the slots (-1: skip)."""
        i = 0
        while i < len(slots):
            if slots[i] < 0:
                i += 1
                continue
            n = 1
            while i + n < len(slots) and slots[i + n] == slots[i] + n and slots[i + n] // self.S == slots[i] // self.S:
                n += 1
            blk, off = slots[i] // self.S, slots[i] % self.S
            pg, bl = blk // self.blocks, blk % self.blocks
            for kind in (0, 1):
                for g in range(self.Hkv):
                    live = self.c[kind][pg, g, bl, :off]
                    y, e = ref64.write_block(live, float(self.e[pg, g, bl, kind]), rows[kind][i:i + n, g])
                    self.c[kind][pg, g, bl, :off + n] = y
                    self.e[pg, g, bl, kind] = e
            i += n

    def check(self, kv):
        other = Blocks(kv)
        for kind in (0, 1):
            assert np.array_equal(other.c[kind], self.c[kind])
        assert np.array_equal(other.e, self.e)


def rows(n, Hkv, seed, dtype=torch.bfloat16, spread=3.0):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn((2, n, Hkv, 128), generator=g, device="cuda")
    x *= torch.exp2(spread * torch.randn((2, n, Hkv, 1), generator=g, device="cuda"))
    return x[0].to(dtype), x[1].to(dtype)


def f64(kv):
    return [x.double().cpu().numpy() for x in kv]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hkv,page,S", [(1, 32, 32), (3, 64, 32), (8, 64, 64), (2, 128, 128), (5, 256, 64)])
def test_prompts_then_tokens(P, dtype, Hkv, page, S):
    lens = [1, page, 0, page + 1, 2 * S - 1, 77]
    B, per = len(lens), 4 + 300 // page
    t = P.PageTables(B, page, per, B * per)
    kv = P.BlockKV(B * per, Hkv, page, S)
    ref = Blocks(kv)
    _, slots, _ = t.plan(i32([0] * B), i32(lens), sum(lens))
    k, v = rows(sum(lens), Hkv, 1, dtype)
    st = i32([0])
    kv.write(k, v, slots, dev_status=st)
    ref.write(f64((k, v)), slots.tolist())
    ref.check(kv)
    # single tokens, larger and smaller than what is there: live rows are coded anew
    for n in range(3):
        _, slots, _ = t.plan(i32([x + n for x in lens]), i32([1] * B), B, 1)
        k, v = rows(B, Hkv, 10 + n, dtype, spread=6.0)
        kv.write(k, v, slots, dev_status=st)
        ref.write(f64((k, v)), slots.tolist())
        ref.check(kv)
    assert st.item() == 0


@pytest.mark.parametrize("T", [1, 7, 64, 100])
def test_tree_rows_and_commit(P, T):
    B, Hkv, page, S, lens = 5, 2, 64, 32, [3, 64, 100, 31, 0]
    t = P.PageTables(B, page, 8, 40)
    kv = P.BlockKV(40, Hkv, page, S)
    ref = Blocks(kv)
    _, slots, _ = t.plan(i32([0] * B), i32(lens), sum(lens))
    p = rows(sum(lens), Hkv, 1)
    kv.write(*p, slots)
    ref.write(f64(p), slots.tolist())
    r = random.Random(T)
    st = i32([0])
    for n in range(3):
        _, slots, _ = t.plan(i32(lens), i32([T] * B), B * T, T)
        x = rows(B * T, Hkv, 20 + n)
        kv.write(*x, slots, dev_status=st)
        ref.write(f64(x), slots.tolist())
        ref.check(kv)
        acc = [sorted(r.sample(range(T), r.randint(0, min(T, 5)))) for _ in range(B)]
        nodes = [a + [-1] * (T - len(a)) for a in acc]
        _, slots, _ = t.plan(i32(lens), i32([len(a) for a in acc]), B * T, T)
        kv.write(*x, slots, src=i32(nodes), rows_per_seq=T, dev_status=st)
        at = [b * T + max(a, 0) for b in range(B) for a in nodes[b]]
        ref.write([y[at] for y in f64(x)], slots.tolist())
        ref.check(kv)
        lens = [a + len(c) for a, c in zip(lens, acc)]
    assert st.item() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_size_of_scale(P, dtype):
    # amax just below, at and above 448 * 2^e; the ends of the format; all zero
    kv = P.BlockKV(4, 2, 128, 32)
    ref = Blocks(kv)
    tops = [448.0, 450.0, 446.0, 1.75, 1.7578125, 0.0, 2.0 ** -125, 2.0 ** 119, 3.0e38, 1e-30, 0.4375, 1.0, 2.0 ** -110, 7.0, 7.03125, 2.0 ** 127]
    k = torch.zeros((16 * 32, 2, 128), device="cuda")
    for i, top in enumerate(tops):
        g = torch.Generator("cuda").manual_seed(i)
        k[32 * i:32 * i + 32] = (torch.rand((32, 2, 128), generator=g, device="cuda") * 2 - 1) * top
        k[32 * i + 5, :, 7] = -top
    k = k.to(dtype)
    v = (-k).flip(2).contiguous()
    st = i32([0])
    kv.write(k, v, torch.arange(512, dtype=torch.int32, device="cuda"), dev_status=st)
    ref.write(f64((k, v)), list(range(512)))
    ref.check(kv)
    assert st.item() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ties_round_to_even(P, dtype):
    # halves between two codes, at every exponent of the format (scale 1: amax 448)
    kv = P.BlockKV(1, 1, 32, 32)
    k = torch.zeros((32, 1, 128), device="cuda")
    x = [448.0]
    for e in range(-9, 9):
        step = 2.0 ** (max(e, -6) - 3)
        x += [s * (2.0 ** e + (m + 0.5) * step) for m in range(8) for s in (1, -1) if 2.0 ** e + (m + 0.5) * step < 440]
    k.view(-1)[:len(x)] = torch.tensor(x)
    k = k.to(dtype)
    assert (k.double().view(-1)[:len(x)].cpu() == torch.tensor(x, dtype=torch.float64)).all()
    ref = Blocks(kv)
    kv.write(k, k, torch.arange(32, dtype=torch.int32, device="cuda"))
    ref.write(f64((k, k)), list(range(32)))
    ref.check(kv)
    assert (kv.scales == 127).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_not_finite(P, dtype):
    for what in (float("inf"), -float("inf"), float("nan")):
        kv = P.BlockKV(1, 2, 64, 64)
        k, v = rows(64, 2, 5, dtype)
        v[9, 1, 3] = what
        ref = Blocks(kv)
        st = i32([0])
        kv.write(k, v, torch.arange(64, dtype=torch.int32, device="cuda"), dev_status=st)
        ref.write(f64((k, v)), list(range(64)))
        ref.check(kv)
        assert st.item() == 14


def test_dead_rows_and_other_pages_stay(P):
    kv = P.BlockKV(3, 2, 64, 32)
    for x in (kv.k_pages, kv.v_pages):
        x.copy_(torch.randint(0, 0x7F, x.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(2)).to(torch.uint8))
    ref = Blocks(kv)
    k, v = rows(4, 2, 7)
    slots = [-1, 64 + 10, 64 + 11, -1]
    kv.write(k, v, i32(slots))
    ref.write(f64((k, v)), slots)
    ref.check(kv)


def test_refused_slots(P):
    k, v = rows(6, 2, 7)
    for slots, status, kept in (([0, 1, 64 * 3, 2, 3, 4], 10, [0, 1]), ([0, 1, -2, 64, 65, 66], 10, [0, 1, -1, 64, 65, 66]),
                                ([0, 1, 3, 64, 65, 66], 13, [0, 1, -1, 64, 65, 66]), ([5, 5, 6, 64, 65, 66], 13, [5, -1, -1, 64, 65, 66])):
        kv = P.BlockKV(3, 2, 64, 32)
        ref = Blocks(kv)
        st = i32([0])
        kv.write(k, v, i32(slots), dev_status=st)
        assert st.item() == status, slots
        if len(kept) == 6:
            ref.write(f64((k, v)), kept)
            ref.check(kv)
    kv = P.BlockKV(3, 2, 64, 32)
    for src in ([0, 3, 1, 0, 1, 2], [0, -1, 1, 0, 1, 2]):
        st = i32([0])
        kv.write(k, v, i32([0, 1, 2, 64, 65, 66]), src=i32(src), rows_per_seq=3, dev_status=st)
        assert st.item() == 13


def test_strided_rows_and_graph(P):
    kv, other = P.BlockKV(4, 2, 64, 32), P.BlockKV(4, 2, 64, 32)
    x = torch.randn((70, 8, 128), device="cuda").bfloat16()  # q, k, v of one projection
    k, v = x[:, 4:6], x[:, 6:]
    slots = torch.arange(30, 100, dtype=torch.int32, device="cuda")
    kv.write(k, v, slots)
    other.write(k.contiguous(), v.contiguous(), slots)
    assert torch.equal(kv.k_pages, other.k_pages) and torch.equal(kv.scales, other.scales)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kv.write(k, v, slots)
    for r in range(3):
        x.copy_(torch.randn(x.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(r)))
        g.replay()
        other.write(k.contiguous(), v.contiguous(), slots)
        torch.cuda.synchronize()
        for a, b in ((kv.k_pages, other.k_pages), (kv.v_pages, other.v_pages), (kv.scales, other.scales)):
            assert torch.equal(a, b)


def test_pages_held_twice_are_reported(P):
    # the free list takes no more than there are pages, and nothing behind it is written
    t = P.PageTables(3, 64, 4, 8)
    wide = torch.full((32,), -7, dtype=torch.int32, device="cuda")
    wide[:8] = t.free_pages
    t.free_pages = wide[:8]
    t.page_table.fill_(5)
    t.num_held.fill_(4)
    t.num_free.fill_(1)
    st = i32([0])
    t.plan(i32([0, 0, 0]), i32([0, 0, 0]), 0, 0, st)
    assert st.item() == 10 and t.num_free.item() == 8
    assert wide[:8].tolist() == [7] + [5] * 7 and (wide[8:] == -7).all()
    assert t.num_held.tolist() == [0, 0, 0]


def test_as_many_rows_as_there_can_be(P):
    # 2^31 - 1 rows of slots: the last workgroup's next row would be past 32 bits
    t = P.PageTables(2, 64, 4, 8)
    N = 2 ** 31 - 1
    slots, start, st = torch.full((N,), 7, dtype=torch.int32, device="cuda"), i32([0, 0, 0]), i32([0])
    P.ptd_page_plan(t.state(), i32([0, 0]), i32([70, 3]), N, 0, start, slots, None, st)
    assert st.item() == 0 and start.tolist() == [0, 70, 73]
    assert slots[:74].tolist() == list(range(70)) + [128, 129, 130, -1]
    assert slots[74:].amax().item() == -1 and slots[74:].amin().item() == -1
