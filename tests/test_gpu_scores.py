"""GPU checks of tree attention at scores far from ordinary ones, over every kind of cache,
against a plain 64-bit implementation.

Large scores.  Every key of a row scores the same 2^22 .. 2^23, and a few score 10 or 12 more,
so that references move and the states of key groups and of splits differ.  Scores
are whole numbers below 2^24, exact in fp32, and so are the caches' values in every
format: what is rounded are the weights.  A weight's exponent is one rounding of s c - R (R the
rounded product of the reference maximum and c, the same for all keys), a number below 2^6: off by
2^-19 at most; the exponential and fp32 sums of positive terms add less than 2^-12 together.
The weights' own rounding to bf16, w (1 + d) with |d| <= 2^-8 above and below the line,
is at most 2^-8 of the average of |v| plus 2^-8 of the output.  So (2^-8 + 2^-11) times the
average and 2^-8 times the output bound every kind; it covers the bf16 outputs' own half step too
where the weights are carried with twice the bits, and fp32 outputs are asked for here."""
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


def attend(P, kind, q, k, v, n, parent, scale, page=64, S=32):
    """k, v [B][Hkv][rows][128] in a cache of `kind`; keys of 8-bit caches are multiples of 16
    times a code."""
    B, Hkv, L, D = k.shape
    args = dict(out_dtype=torch.float32, scale=scale)
    e4 = lambda x: x.to(torch.float8_e4m3fn).view(torch.uint8)
    if kind == "bf16":
        return P.tree_attention(q, k, v, i32(n), i32(parent), **args)
    sixteen = torch.full((Hkv,), 16.0, device="cuda")
    if kind == "fp8kv":
        return P.tree_attention_fp8kv(q, e4(k / 16), e4(v), sixteen, None, i32(n), i32(parent), **args)
    per = L // page
    table = np.random.default_rng(L).permutation(B * per).reshape(B, per)

    def pages(x):
        got = torch.empty((B * per, Hkv, page, D), dtype=x.dtype, device="cuda")
        got[torch.from_numpy(table).cuda().flatten()] = x.unflatten(2, (per, page)).transpose(1, 2).flatten(0, 1)
        return got

    if kind == "paged":
        return P.tree_attention_paged(q, pages(k), pages(v), i32(table), i32(n), i32(parent), **args)
    if kind == "paged_fp8kv":
        return P.tree_attention_paged(q, pages(e4(k / 16)), pages(e4(v)), i32(table), i32(n), i32(parent),
                                      k_scale=sixteen, **args)
    kv = P.BlockKV(B * per, Hkv, page, S)
    kv.k_pages.copy_(pages(e4(k / 16)))
    kv.v_pages.copy_(pages(e4(v)))
    kv.scales[..., 0] = 131
    return kv.tree_attention(q, i32(table), i32(n), i32(parent), **args)


KINDS = ["bf16", "paged", "fp8kv", "paged_fp8kv", "fp8blk"]


# rows per head 4, 128, 256 of one sequence (four, four and two key groups) and of several (one)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,T,Hq,Hkv,n", [(1, 1, 8, 2, 190), (1, 1, 8, 2, 5000), (1, 64, 4, 2, 1500), (1, 64, 8, 2, 200),
                                          (1, 64, 8, 2, 6000), (3, 64, 8, 2, 700), (16, 64, 8, 2, 2900)])
def test_large_scores(P, kind, B, T, Hq, Hkv, n):
    L = (n + T + 63) // 64 * 64
    r = np.random.default_rng(n + T)
    lens = [n - 7 * b for b in range(B)]
    k = torch.zeros((B, Hkv, L, 128), device="cuda")
    v = torch.full_like(k, 0.5)
    k[..., 0] = 4096
    for b in range(B):
        tens = torch.from_numpy(r.choice(lens[b], lens[b] // 32, replace=False)).cuda()
        k[b, :, tens, 1], v[b, :, tens] = 10, -1
        for at in (lens[b] - 1, int(r.integers(lens[b]))):
            k[b, :, at, 1], v[b, :, at] = 12, 1
    q = torch.zeros((B, T, Hq, 128), device="cuda")
    # another product for each row: 1024 .. 2040 in steps of 8, exact in bf16
    q[..., 0] = (torch.arange(B * T * Hq, device="cuda") * 8 % 1024 + 1024).float().view(B, T, Hq)
    q[..., 1] = 1
    parent = np.stack([W.tree_uniform(r, T)[0] for _ in range(B)])
    q, k, v = (x.bfloat16() for x in (q, k, v))
    out = attend(P, kind, q, k, v, lens, parent, 1.0).double()
    for b in range(B):
        ref, mag = ref64.tree(q[b], k[b], v[b], lens[b], parent[b], 1.0, T)
        assert ((out[b] - ref).abs() <= (2.0 ** -8 + 2.0 ** -11) * mag + 2.0 ** -8 * ref.abs()).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,T", [(1, 100), (2, 200)])
def test_large_scale(P, kind, B, T):
    # a scale of 2^29 on products of about 2^-29, and rows whose first keys are other branches'
    Hq, Hkv, scale = 4, 2, 2.0 ** 29
    L = (T + 63) // 64 * 64
    g = torch.Generator("cuda").manual_seed(T)
    q = (torch.randn((B, T, Hq, 128), generator=g, device="cuda") * 2.0 ** -34).bfloat16()
    k = (torch.randint(-8, 9, (B, Hkv, L, 128), generator=g, device="cuda") * 2.0).bfloat16()
    v = torch.randint(-8, 9, (B, Hkv, L, 128), generator=g, device="cuda").bfloat16()
    parent = np.stack([W.tree_star(T)[0]] * B)
    out = attend(P, kind, q, k, v, [0] * B, parent, scale).double()
    for b in range(B):
        ref, mag = ref64.tree(q[b], k[b], v[b], 0, parent[b], scale, T)
        assert ((out[b] - ref).abs() <= (2.0 ** -8 + 2.0 ** -11) * mag + 2.0 ** -8 * ref.abs()).all()
