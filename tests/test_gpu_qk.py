"""GPU checks of ptd_qk_norm_rope: norm, rotation and rows into the caches against a plain
64-bit implementation.

Errors of fp32: the sum of squares adds 16 elements and 3 steps (19 * 2^-24, halved by the
root), mean, eps, root, reciprocal and the two products of the norm add at most 8 * 2^-24, cosine and sine,
two products and their sum at most 4 * 2^-24 of |u| + |v| of the pair: below 2^-19 of it in all. A bf16
output is rounded once more, by up to 2^-8 of itself."""
import pytest
import torch

import ref64_samples as R

pytestmark = pytest.mark.gpu
FP32 = 2.0 ** -19


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_10661_amd as lib
    return lib


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def near(got, ref, mag):
    tol = FP32 * mag + (2.0 ** -8 * ref.abs() if got.dtype == torch.bfloat16 else 2.0 ** -24 * ref.abs())
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bad.any(), (bad.nonzero()[:3].tolist(), ((got.double() - ref).abs() / tol.clamp(min=1e-300)).max().item())


def freqs(theta, rot):
    return [theta ** (-2.0 * p / rot) for p in range(rot // 2)]


def rows(N, Hq, Hkv, D, dtype, fused, seed=0):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn((N, Hq + 2 * Hkv, D), generator=g, device="cuda") * torch.exp(2 * torch.randn((N, Hq + 2 * Hkv, 1), generator=g, device="cuda"))
    x = x.to(dtype)
    got = (x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:])
    return got if fused else tuple(y.contiguous() for y in got)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,rot", [(128, 128), (128, 64), (128, 16), (128, 112), (64, 64), (64, 32), (64, 48), (64, 0)])
@pytest.mark.parametrize("inter", [False, True])
def test_norm_and_rotation(P, dtype, D, rot, inter):
    for n, (N, Hq, Hkv, norm) in enumerate([(1, 32, 8, True), (5, 7, 1, True), (130, 28, 4, True), (33, 1, 1, False), (64, 17, 17, True)]):
        q, k, _ = rows(N, Hq, Hkv, D, dtype, fused=n % 2 == 0, seed=n)
        g = torch.Generator("cuda").manual_seed(99 + n)
        pos = torch.randint(0, 200000, (N,), generator=g, device="cuda", dtype=torch.int32)
        wd = [dtype, torch.float32, torch.bfloat16][n % 3]
        wq, wk = (torch.randn(D, generator=g, device="cuda").to(wd) for _ in range(2)) if norm else (None, None)
        if n == 4:
            wk = None
        st = i32([0])
        eps = 1e-5 if norm else None
        oq, ok = P.qk_norm_rope(q, k, pos, wq, wk, eps=eps, rot_dim=rot, theta=10000.0,
                                pairing=P.PTD_ROPE_INTERLEAVED if inter else P.PTD_ROPE_HALF, dev_status=st)
        f = freqs(10000.0, rot)
        for got, x, w in ((oq, q, wq), (ok, k, wk)):
            near(got, *R.heads(x, w, pos, f, rot, inter, eps))
        assert st.item() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,Hkv,D", [(32, 8, 128), (1, 2, 64), (100, 3, 128), (256, 1, 64)])
def test_rows_into_pages(P, dtype, page, Hkv, D):
    N, Hq, num = 77, Hkv * 2, 200 // page + 90 // min(page, 64) + 2
    q, k, v = rows(N, Hq, Hkv, D, dtype, fused=True, seed=page)
    r = torch.Generator().manual_seed(page)
    slots = torch.randperm(num * page, generator=r)[:N].int()
    slots[::7] = -1
    pos = torch.arange(N, dtype=torch.int32) * 3
    pos[3], pos[70] = -1, -5
    kp, vp = (torch.full((num, Hkv, page, D), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    oq, ok = torch.full((N, Hq, D), 9.0, dtype=dtype, device="cuda"), torch.full((N, Hkv, D), 9.0, dtype=dtype, device="cuda")
    w = torch.rand(D, device="cuda").to(dtype)
    st = i32([0])
    P.qk_norm_rope(q, k, pos.cuda(), w, w, v=v, slots=slots.cuda(), k_pages=kp, v_pages=vp, q_out=oq, k_out=ok, dev_status=st)
    assert st.item() == 0
    there = (pos >= 0)
    f = freqs(10000.0, D)
    for got, x in ((oq, q), (ok, k)):
        ref, mag = R.heads(x, w, pos.cuda(), f, D, False, 1e-6)
        near(got[there], ref[there], mag[there])
        assert (got[~there] == 9).all()
    # the pages hold the very outputs, and nothing else changed
    wk, wv = torch.full_like(kp, 7.0), torch.full_like(vp, 7.0)
    for i in range(N):
        if there[i] and slots[i] >= 0:
            wk[slots[i] // page, :, slots[i] % page] = ok[i]
            wv[slots[i] // page, :, slots[i] % page] = v[i]
    assert torch.equal(kp, wk) and torch.equal(vp, wv)


def test_pages_alone_and_contiguous_cache(P):
    # no k_out: the rows go to the cache [B][Hkv][L_cap][D] only, which is B pages of L_cap rows
    B, T, Hq, Hkv, D, L = 3, 5, 4, 2, 64, 37
    q, k, v = rows(B * T, Hq, Hkv, D, torch.float32, fused=False)
    kv = [0, 11, 32]
    pos = i32([kv[b] + t for b in range(B) for t in range(T)])
    slots = i32([b * L + kv[b] + t for b in range(B) for t in range(T)])
    kc, vc = (torch.zeros((B, Hkv, L, D), device="cuda") for _ in range(2))
    oq = torch.empty_like(q)
    shape = P.QKShape(B * T, Hq, Hkv, D, D, P.PTD_ROPE_HALF, 1, P.PTD_F32, P.PTD_F32, 0, 0, 0, 0, 0, 1e-6, 10000.0)
    P.ptd_qk_norm_rope(q, k, v, None, None, pos, slots, oq, None, P.KVStore(kc.data_ptr(), vc.data_ptr(), L, B), shape)
    ref, mag = R.heads(k, None, pos, freqs(10000.0, D), D, False, 1e-6)
    for b in range(B):
        at = slice(b * T, (b + 1) * T)
        near(kc[b, :, kv[b]:kv[b] + T].transpose(0, 1), ref[at], mag[at])
        assert torch.equal(vc[b, :, kv[b]:kv[b] + T].transpose(0, 1), v[at])
    assert (kc != 0).sum() == (vc != 0).sum() == B * T * Hkv * D


def test_agrees_with_tree_rope(P):
    # without the norm it is the rotation that tree rows in contiguous caches get
    B, T, Hq, Hkv, D, L = 2, 16, 4, 2, 128, 64
    g = torch.Generator("cuda").manual_seed(1)
    parent = i32([[-1] + [i // 2 for i in range(T - 1)]] * B)
    kv = i32([0, 40])
    for dtype in (torch.bfloat16, torch.float32):
        q = torch.randn((B, T, Hq, D), generator=g, device="cuda").to(dtype)
        kc = torch.randn((B, Hkv, L, D), generator=g, device="cuda").to(dtype)
        k = torch.stack([kc[b, :, kv[b]:kv[b] + T].transpose(0, 1) for b in range(B)]).reshape(B * T, Hkv, D).contiguous()
        q0 = q.clone()
        pos = P.tree_rope(q, kc, kv, parent)
        oq, ok = P.qk_norm_rope(q0.view(B * T, Hq, D), k, pos.view(-1), eps=None)
        turned = torch.stack([kc[b, :, kv[b]:kv[b] + T].transpose(0, 1) for b in range(B)]).reshape(B * T, Hkv, D)
        for got, want in ((oq, q.view(B * T, Hq, D)), (ok, turned)):
            # both round the exact value's fp32 neighbour: a step of the type apart at most
            eps = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -22
            assert ((got.double() - want.double()).abs() <= eps * want.double().abs() + 2e-6).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_in_place(P, dtype):
    N, Hq, Hkv, D = 50, 9, 3, 128
    for inter in (P.PTD_ROPE_HALF, P.PTD_ROPE_INTERLEAVED):
        q, k, v = rows(N, Hq, Hkv, D, dtype, fused=True, seed=4)
        pos = torch.arange(N, dtype=torch.int32, device="cuda") * 1000
        oq, ok = P.qk_norm_rope(q, k, pos, rot_dim=96, pairing=inter)
        keep = v.clone()
        a, b = P.qk_norm_rope(q, k, pos, rot_dim=96, pairing=inter, q_out=q, k_out=k)
        assert a is q and b is k
        assert torch.equal(q, oq) and torch.equal(k, ok) and torch.equal(v, keep)


def test_far_positions_and_own_frequencies(P):
    # angles of positions up to 2^31 - 1: the turned pair is exact to fp32, whatever the angle
    pos = i32([0, 1, 2 ** 20 + 1, 10 ** 8, 2 ** 31 - 1, 2 ** 31 - 2])
    q, k, _ = rows(6, 2, 1, 128, torch.float32, fused=False)
    f = [1.0, -0.5, 3.75, 1024.0, 1e-9, 0.0, 2.0 ** 20] + freqs(5e5, 128)[7:]
    oq, ok = P.qk_norm_rope(q, k, pos, eps=None, inv_freq=f)
    for got, x in ((oq, q), (ok, k)):
        near(got, *R.heads(x, None, pos, f, 128, False, None))
    assert torch.equal(oq[0], q[0])  # position 0 turns nothing


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_odd_values_stay_in_their_head(P, dtype):
    N, Hq, Hkv, D = 6, 5, 2, 128
    q, k, v = rows(N, Hq, Hkv, D, dtype, fused=False)
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    want, wk = P.qk_norm_rope(q, k, pos)
    q[1, 2, 5], q[2, 0, 100], q[3, 4] = float("nan"), float("inf"), 0.0
    k[4, 1, 0] = float("-inf")
    got, gk = P.qk_norm_rope(q, k, pos)
    got0, _ = P.qk_norm_rope(q, k, pos, eps=0.0)
    hit = torch.zeros((N, Hq), dtype=torch.bool, device="cuda")
    hit[1, 2] = hit[2, 0] = hit[3, 4] = True
    assert torch.equal(got[~hit], want[~hit])
    assert got[1, 2].isnan().all() and got[2, 0, [36, 100]].isnan().all() and (got[2, 0].nan_to_num() == 0).all()
    assert (got[3, 4] == 0).all() and got0[3, 4].isnan().all()  # a head of zeros: eps keeps it
    assert torch.equal(gk[:4], wk[:4]) and torch.equal(gk[5], wk[5]) and torch.equal(gk[4, 0], wk[4, 0])
    # small and large heads: the sum of squares is fp32
    for size in (1e-18, 1e-10, 1e10, 1e18):
        x = (torch.randn((3, 2, D), device="cuda") * size).to(dtype)
        a, b = P.qk_norm_rope(x, x, pos[:3], eps=0.0)
        near(a, *R.heads(x, None, pos[:3], freqs(10000.0, D), D, False, 0.0))


def test_bad_slots_are_reported(P):
    N, Hkv, D, page, num = 4, 2, 64, 32, 3
    q, k, v = rows(N, 2, Hkv, D, torch.float32, fused=False)
    for bad in (page * num, 2 ** 31 - 1, -2, -2 ** 31):
        kp, vp = (torch.zeros((num + 1, Hkv, page, D), device="cuda") for _ in range(2))
        st = i32([0])
        P.qk_norm_rope(q, k, i32([0, 1, 2, 3]), v=v, slots=i32([5, bad, -1, 7]), k_pages=kp[:num], v_pages=vp[:num], dev_status=st)
        assert st.item() == 10
        assert vp.view(-1, D).ne(0).any(1).sum() == 2 * Hkv
        assert torch.equal(vp[0, :, 5], v[0]) and torch.equal(vp[0, :, 7], v[3])


def test_one_kind_of_heads(P):
    N, D = 9, 128
    q, k, _ = rows(N, 6, 2, D, torch.bfloat16, fused=False)
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    wq, wk = P.qk_norm_rope(q, k, pos)
    oq, ok = torch.zeros_like(q), torch.zeros_like(k)
    s = lambda Hq, Hkv: P.QKShape(N, Hq, Hkv, D, D, P.PTD_ROPE_HALF, 1, P.PTD_BF16, P.PTD_BF16, 0, 0, 0, 0, 0, 1e-6, 10000.0)  # noqa: E731
    P.ptd_qk_norm_rope(q, None, None, None, None, pos, None, oq, None, None, s(6, 0))
    P.ptd_qk_norm_rope(None, k, None, None, None, pos, None, None, ok, None, s(0, 2))
    assert torch.equal(oq, wq) and torch.equal(ok, wk)


def test_graph_and_other_stream(P):
    N, Hq, Hkv, D, page = 40, 8, 2, 128, 64
    q, k, v = rows(N, Hq, Hkv, D, torch.bfloat16, fused=True)
    base = q._base if q._base is not None else q
    pos, slots = torch.arange(N, dtype=torch.int32, device="cuda"), torch.arange(N, dtype=torch.int32, device="cuda") + 30
    kp, vp = (torch.zeros((2, Hkv, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    oq, ok = torch.empty((N, Hq, D), dtype=torch.bfloat16, device="cuda"), torch.empty((N, Hkv, D), dtype=torch.bfloat16, device="cuda")
    kw = dict(v=v, slots=slots, k_pages=kp, v_pages=vp)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.qk_norm_rope(q, k, pos, q_out=oq, k_out=ok, **kw)
    for r in range(3):
        base.copy_(torch.randn(base.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(r)))
        pos.copy_(torch.arange(N, dtype=torch.int32) + 100 * r)
        g.replay()
        torch.cuda.synchronize()
        a, b = P.qk_norm_rope(q, k, pos)
        assert torch.equal(a, oq) and torch.equal(b, ok) and torch.equal(kp.transpose(1, 2).reshape(-1, Hkv, D)[30:70], ok)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a, b = P.qk_norm_rope(q, k, pos)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(a, oq) and torch.equal(b, ok)


def test_many_rows(P):
    # more rows than one round of waves; each row equals the row by itself
    N, Hq, Hkv, D = 20011, 4, 1, 64
    q, k, _ = rows(N, Hq, Hkv, D, torch.bfloat16, fused=True)
    pos = torch.randint(0, 10 ** 6, (N,), dtype=torch.int32, device="cuda")
    oq, ok = P.qk_norm_rope(q, k, pos)
    near(oq, *R.heads(q, None, pos, freqs(10000.0, D), D, False, 1e-6))
    a, b = P.qk_norm_rope(q[20010:], k[20010:], pos[20010:].contiguous())
    assert torch.equal(a[0], oq[20010]) and torch.equal(b[0], ok[20010])
