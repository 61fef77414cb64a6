"""GPU checks of ptd_prompt_attention against a plain 64-bit implementation.

Bounds.  bf16 inputs: the softmax weights w are rounded to bf16, w (1 + d) with |d| at most
half a step, 2^-8, and so is their sum, 1 + D, D the mean of d: an output is off by (sum w d
v - D out) / (1 + D), at most 2^-8 of the average of |v| plus 2^-8 of the output; 2^-11
of the average more covers fp32 sums and exponentials, and bf16 outputs add their
own half step, 2^-8 of the output.  fp32 inputs: a weight's relative error is
that of its score (D roundings of 2^-24 of scale * sum |q k|, twice for the reference
maximum) and of the exponential (its argument rounded at most at 2^-23 of itself, and
four units); the sums over n keys add n roundings."""
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


def starts_of(lens):
    return [sum(lens[:i]) for i in range(len(lens) + 1)]


def inputs(lens, Hq, Hkv, D, dtype, seed=0, fused=False, amp=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    N = sum(lens)
    if fused:
        x = torch.randn((N, Hq + 2 * Hkv, D), generator=g, device="cuda").to(dtype)
        return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    q, k, v = (torch.randn((N, h, D), generator=g, device="cuda") for h in (Hq, Hkv, Hkv))
    return (q * amp).to(dtype), k.to(dtype), v.to(dtype)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def bound(ref, mag, top, n, D, dtype, out_dtype):
    if dtype == torch.bfloat16:
        tol = (2.0 ** -8 + 2.0 ** -11) * mag + 2.0 ** -8 * ref.abs()
    else:
        tol = 2.0 ** -24 * ((4 * D + 4) * top[..., None] + n + 16) * mag
    if out_dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * ref.abs()
    return tol + 1e-30


def check(P, lens, Hq, Hkv, D, dtype=torch.bfloat16, out_dtype=None, fused=False, amp=1.0, scale=0.0, seed=0):
    q, k, v = inputs(lens, Hq, Hkv, D, dtype, seed, fused, amp)
    st = i32([0])
    starts = starts_of(lens)
    out = P.prompt_attention(q, k, v, i32(starts), out_dtype=out_dtype, scale=scale, dev_status=st)
    assert st.item() == 0
    ref, mag, top = ref64.causal(q, k, v, starts, scale or 1.0 / np.sqrt(D))
    err = (out.double() - ref).abs() - bound(ref, mag, top, max(lens), D, dtype, out.dtype)
    assert err.max() <= 0, err.max().item()
    return out


@pytest.mark.parametrize("n", [1, 2, 15, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 511, 513])
def test_lengths(P, n):
    check(P, [n], 4, 2, 128, out_dtype=torch.float32, seed=n)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 8), (8, 1), (6, 3), (5, 5), (14, 2), (32, 8), (40, 40), (3, 1)])
@pytest.mark.parametrize("D", [64, 128])
def test_heads(P, Hq, Hkv, D):
    check(P, [37, 130], Hq, Hkv, D, out_dtype=torch.float32, fused=Hq % 2 == 0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_packed(P, dtype, D):
    # empty prompts at both ends and between, single tokens, more sequences than lanes
    check(P, [0, 0, 5, 1, 0, 64, 300, 1, 1, 129, 0], 4, 2, D, dtype)
    check(P, [(7 * i) % 11 for i in range(150)], 4, 4, D, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_long(P, dtype):
    check(P, [2000, 17, 1100], 8, 2, 128, dtype, fused=True)
    check(P, [4097], 2, 1, 64, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_scores_far_apart(P, dtype):
    # scores of +-100 and more: the reference maximum moves late and often
    check(P, [700, 90], 4, 2, 128, dtype, out_dtype=torch.float32, amp=12.0)
    check(P, [400], 2, 2, 64, dtype, out_dtype=torch.float32, scale=2.5)


def test_rising_scores(P):
    # every key scores higher than all before it: the reference moves in every tile
    n, D = 600, 128
    q = torch.ones((n, 2, D), device="cuda", dtype=torch.bfloat16)
    k = (torch.arange(n, device="cuda").float()[:, None, None].expand(n, 1, D) / 8).bfloat16().contiguous()
    v = torch.randn((n, 1, D), device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
    out = P.prompt_attention(q, k, v, i32([0, n]), out_dtype=torch.float32)
    ref, mag, top = ref64.causal(q, k, v, [0, n], D ** -0.5)
    assert ((out.double() - ref).abs() <= bound(ref, mag, top, n, D, torch.bfloat16, torch.float32)).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_low_scores(P, dtype):
    # equal scores of about -8e6: the plain mean (the product of the reference maximum
    # and the scale is rounded at 2^-24 of itself, the same for every key)
    D, n = 64, 70
    q, k, v = inputs([n], 2, 1, D, dtype)
    q, k = torch.full_like(q, -1024.0), torch.full_like(k, 1024.0)
    out = P.prompt_attention(q, k, v, i32([0, n]), out_dtype=torch.float32)
    ref, mag, _ = ref64.causal(q, k, v, [0, n], D ** -0.5)
    assert ((out.double() - ref).abs() <= 2.0 ** -24 * (n + 16) * mag).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [64, 200, 450])
def test_huge_scores(P, dtype, n):
    # scores of up to 2^23, exact in fp32: a few keys 10 above the first one, 0 elsewhere, then one 12
    # above it, so that the weights of the keys before count beside its own
    D = 64
    q, k, v = (torch.zeros((n, 1, D), device="cuda") for _ in range(3))
    q[:, 0, 0] = (8 * torch.arange(n, device="cuda") % 1024 + 1024).float()
    q[:, 0, 1] = 1
    k[:, 0, 0] = 4096
    k[32:n - 1:32, 0, 1] = 10
    k[n - 1, 0, 1] = 12
    v[n - 1] = 1
    q, k, v = (torch.cat([x] * 20).to(dtype) for x in (q, k, v))
    for s in range(20):  # another product for each of the last rows
        q[(s + 1) * n - 1, 0, 0] = 1024 + 8 * s
    starts = starts_of([n] * 20)
    out = P.prompt_attention(q, k, v, i32(starts), out_dtype=torch.float32, scale=1.0)
    ref, mag, _ = ref64.causal(q, k, v, starts, 1.0)
    assert ((out.double() - ref).abs() <= (2.0 ** -8 + 2.0 ** -11) * mag + 2.0 ** -8 * ref.abs()).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("at", [0, 70, 129])
@pytest.mark.parametrize("what", [float("inf"), -float("inf"), float("nan")])
def test_what_is_not_seen_does_not_matter(P, dtype, at, what):
    lens, D = [130, 40], 128
    q, k, v = inputs(lens, 4, 2, D, dtype)
    clean = P.prompt_attention(q, k, v, i32(starts_of(lens)))
    k2, v2 = k.clone(), v.clone()
    k2[at], v2[at, :, 3] = what, what
    out = P.prompt_attention(q, k2, v2, i32(starts_of(lens)))
    same = torch.ones(170, dtype=torch.bool, device="cuda")
    same[at:130] = False
    assert torch.equal(out[same], clean[same])
    # a value alone: its column is what it is for the rows that see it, the rest is untouched
    out = P.prompt_attention(q, k, v2, i32(starts_of(lens)))
    assert torch.equal(out[same], clean[same])
    seen = out[at:130]
    rest = [d for d in range(D) if d != 3]
    assert torch.equal(seen[..., rest], clean[at:130][..., rest])
    assert seen[..., 3].isnan().all() if np.isnan(what) else (seen[..., 3] == what).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_outside_are_left(P, dtype):
    q, k, v = inputs([400], 4, 2, 128, dtype)
    out = torch.full_like(q, 7.0)
    st = i32([0])
    P.prompt_attention(q, k, v, i32([20, 100, 100, 333]), out=out, dev_status=st)
    assert st.item() == 0
    assert (out[:20] == 7).all() and (out[333:] == 7).all()
    a = P.prompt_attention(q[20:100], k[20:100], v[20:100], i32([0, 80]))
    b = P.prompt_attention(q[100:333], k[100:333], v[100:333], i32([0, 233]))
    assert torch.equal(out[20:100], a) and torch.equal(out[100:333], b)


def test_strides(P):
    # rows wider than their heads, each of q, k, v its own; 16-byte steps only
    lens, D = [90, 41], 64
    N = sum(lens)
    g = torch.Generator("cuda").manual_seed(3)
    bq = torch.randn((N, 4 * D + 8), device="cuda", generator=g).bfloat16()
    bk = torch.randn((N, 2 * D + 24), device="cuda", generator=g).bfloat16()
    bv = torch.randn((N, 2 * D), device="cuda", generator=g).bfloat16()
    q, k = bq[:, 8:].unflatten(1, (4, D)), bk[:, 16:16 + 2 * D].unflatten(1, (2, D))
    v = bv.unflatten(1, (2, D))
    s = i32(starts_of(lens))
    assert torch.equal(P.prompt_attention(q, k, v, s), P.prompt_attention(q.contiguous(), k.contiguous(), v, s))
    with pytest.raises(P.PTDError) as e:  # 8 bytes off
        P.prompt_attention(bq[:, 4:4 + 4 * D].unflatten(1, (4, D)), k, v, s)
    assert e.value.status == 4


def test_bad_starts_are_reported(P):
    q, k, v = inputs([100], 2, 2, 64, torch.bfloat16)
    good = P.prompt_attention(q[:50], k[:50], v[:50], i32([0, 50]))
    for starts in ([0, 50, 40], [0, 50, 101], [-1, 0, 50], [0, 50] + [50] * 90 + [49]):
        st = i32([0])
        out = P.prompt_attention(q, k, v, i32(starts), dev_status=st)
        assert st.item() == 13, starts
        assert torch.equal(out[:50], good)
    # fewer rows than sequences, the wrong one behind all of them
    for dtype in (torch.bfloat16, torch.float32):
        q, k, v = inputs([1], 2, 2, 64, dtype)
        st = i32([0])
        out = P.prompt_attention(q, k, v, i32([0] + [1] * 130 + [2]), dev_status=st)
        assert st.item() == 13 and torch.equal(out, v)


def test_same_results_again_and_alone(P):
    lens = [333, 64, 1000, 5]
    q, k, v = inputs(lens, 8, 2, 128, torch.bfloat16)
    s = starts_of(lens)
    out = P.prompt_attention(q, k, v, i32(s))
    for _ in range(3):
        assert torch.equal(out, P.prompt_attention(q, k, v, i32(s)))
    for a, b in zip(s[:-1], s[1:]):
        assert torch.equal(out[a:b], P.prompt_attention(q[a:b], k[a:b], v[a:b], i32([0, b - a])))


def test_nothing_to_do(P):
    q, k, v = inputs([0], 2, 1, 64, torch.bfloat16)
    assert P.prompt_attention(q, k, v, i32([0, 0])).shape == (0, 2, 64)
    q, k, v = inputs([3], 2, 1, 64, torch.bfloat16)
    assert (P.prompt_attention(q, k, v, i32([2, 2, 2])) == 0).all()


def test_graph_and_streams(P):
    lens = [200, 31]
    q, k, v = inputs(lens, 4, 2, 128, torch.bfloat16)
    s = i32(starts_of(lens))
    want = P.prompt_attention(q, k, v, s)
    out = torch.zeros_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        P.prompt_attention(q, k, v, s, out=out)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.prompt_attention(q, k, v, s, out=out)
    for r in range(3):
        q.copy_(torch.randn(q.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(r)))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, P.prompt_attention(q, k, v, s))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (2, 1), (6, 2), (16, 16), (7, 7), (24, 1)])
def test_many_sequences_of_all_lengths(P, dtype, Hq, Hkv):
    # tiles of several sequences, longest first, whatever the heads' share of the XCDs
    r = np.random.default_rng(Hq)
    check(P, [int(x) for x in r.integers(0, 400, 9)], Hq, Hkv, 64, dtype, seed=Hq)
    check(P, [int(x) for x in r.integers(0, 90, 65)], Hq, Hkv, 64, dtype, seed=Hq + 1)


def test_rows_far_apart(P):
    # 64 rows span more than 2 GiB: offsets beyond 32 bits
    D, n, ld = 64, 70, 1 << 24
    buf = torch.zeros(n * ld, dtype=torch.bfloat16, device="cuda")
    wide = buf.view(n, ld)[:, :D].unflatten(1, (1, D))
    q, k, v = inputs([n], 1, 1, D, torch.bfloat16)
    want = P.prompt_attention(q, k, v, i32([0, n]))
    wide.copy_(v)
    assert torch.equal(P.prompt_attention(q, k, wide, i32([0, n])), want)
    wide.copy_(k)
    assert torch.equal(P.prompt_attention(q, wide, v, i32([0, n])), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_heads_share_a_position(P, dtype):
    # a tile of rows is one position, so the last tile of keys can be seen whole
    check(P, [130, 64, 193], 128, 1, 64, dtype)
    check(P, [129], 96, 1, 128, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale", [0.0, 1.0, 40.0])
@pytest.mark.parametrize("n0", [1, 40, 64, 130])
def test_keys_that_weigh_nothing_come_first(P, dtype, scale, n0):
    # scores of -inf before the first finite one: rows from there on are as if those keys were
    # not there, at any scale
    n, D = 300, 64
    q, k, v = inputs([n], 4, 2, D, dtype, seed=n0)
    q[..., 0] = 1
    k[:n0, :, 0] = -float("inf")
    out = P.prompt_attention(q, k, v, i32([0, n]), out_dtype=torch.float32, scale=scale)[n0:]
    ref, mag, top = ref64.causal(q[n0:], k[n0:], v[n0:], [0, n - n0], scale or D ** -0.5)
    assert ((out.double() - ref).abs() <= bound(ref, mag, top, n, D, dtype, torch.float32)).all()
