"""GPU checks of tree attention over 8-bit pages with block scales
(ptd_tree_attention_paged_fp8blk) against a plain 64-bit implementation on the values that
the pages stand for.  A code times its power-of-two scale is a bf16 number, exactly, so what
is rounded are the softmax weights, above and below the line: w (1 + d) with |d| <= 2^-8,
and their sum by the mean of d, which is at most 2^-8 of the average of |v| plus 2^-8 of
the output; 2^-11 of the average more covers fp32 sums and exponentials, and bf16
outputs add their own half step."""
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


def decode(pages, scales, S):
    x = pages.view(torch.float8_e4m3fn).double().unflatten(2, (-1, S))
    return (x * torch.exp2(scales.double() - 127)[..., None, None]).flatten(2, 3)


def make(P, seed, B, T, Hq, Hkv, page, S, per, kv_len, live=None, spread=2):
    """Pages through a random table, codes of every magnitude, scales that keep the values
    near one; what no row uses holds NaN codes and NaN exponents."""
    g = torch.Generator("cuda").manual_seed(seed)
    r = np.random.default_rng(seed)
    n = B * per + 3
    kv = P.BlockKV(n, Hkv, page, S)
    table = r.permutation(n)[:B * per].reshape(B, per).astype(np.int32)
    for kind, x in enumerate((kv.k_pages, kv.v_pages)):
        e = torch.randint(-spread, spread + 1, (n, Hkv, page // S), generator=g, device="cuda")
        y = torch.randn(x.shape, generator=g, device="cuda").unflatten(2, (-1, S)) * torch.exp2(6.0 - e)[..., None, None]
        x.copy_(y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).flatten(2, 3))
        kv.scales[..., kind] = (127 - 6 + e).to(torch.uint8)
    clean = [decode(x, kv.scales[..., i], S).to(torch.bfloat16) for i, x in enumerate((kv.k_pages, kv.v_pages))]
    used = np.zeros((n, page), bool)
    for b in range(B):
        rows = kv_len[b] + (T if live is None else live[b])
        for p in range(per):
            used[table[b, p], :max(0, min(page, rows - p * page))] = True
    dead = torch.from_numpy(~used).cuda()
    for x in (kv.k_pages, kv.v_pages):
        x.transpose(1, 2)[dead] = 0x7F
    kv.scales.transpose(1, 2)[dead.unflatten(1, (-1, S)).all(2)] = 255
    q = torch.randn((B, T, Hq, 128), generator=g, device="cuda").bfloat16()
    return kv, clean, i32(table), q


def check(P, seed, B, T, Hq, Hkv, page, S, per, kv_len, parent, live=None):
    kv, (kc, vc), table, q = make(P, seed, B, T, Hq, Hkv, page, S, per, kv_len, live)
    st = i32([0])
    tl = None if live is None else i32(live)
    outs = [kv.tree_attention(q, table, i32(kv_len), i32(parent), out_dtype=od, dev_status=st, tree_len=tl).double()
            for od in (torch.bfloat16, torch.float32)]
    assert st.item() == 0
    for b in range(B):
        k, v = (x[table[b].long()].transpose(0, 1).reshape(Hkv, per * page, 128) for x in (kc, vc))
        n = T if live is None else live[b]
        ref, mag = ref64.tree(q[b], k, v, kv_len[b], parent[b], 128 ** -0.5, n)
        tol = (2.0 ** -8 + 2.0 ** -11) * mag + 2.0 ** -8 * ref.abs()
        assert ((outs[1][b] - ref).abs() <= tol).all()
        assert ((outs[0][b] - ref).abs() <= tol + 2.0 ** -8 * (ref.abs() + tol)).all()
        assert (outs[0][b, n:] == 0).all() and (outs[1][b, n:] == 0).all()


@pytest.mark.parametrize("page,S", [(32, 32), (64, 32), (64, 64), (128, 32), (128, 128), (512, 64)])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (4, 4), (3, 3)])
def test_pages_and_scales(P, page, S, Hq, Hkv):
    r = np.random.default_rng(page + S)
    T, per = 13, 1024 // page
    parent = np.stack([W.tree_uniform(r, T)[0] for _ in range(3)])
    check(P, page + S + Hq, 3, T, Hq, Hkv, page, S, per, [0, 300, 1024 - T], parent)


@pytest.mark.parametrize("T", [1, 2, 33, 64, 130, 200])
@pytest.mark.parametrize("B", [1, 2, 3])
def test_tree_sizes(P, T, B):
    r = np.random.default_rng(T)
    parent = np.stack([W.tree_chain(T)[0], W.tree_uniform(r, T)[0], W.tree_star(T)[0]])[:B]
    check(P, T, B, T, 32, 8, 64, 32, 24, [1300, 1536 - T, 0][:B], parent)


def test_single_tokens(P):
    B = 16
    kv = [0, 1, 31, 32, 33, 63, 64, 65, 500, 1000, 2047, 1, 7, 1024, 96, 300]
    check(P, 4, B, 1, 32, 8, 64, 64, 32, kv, np.full((B, 1), -1, np.int32))


def test_ragged(P):
    r = np.random.default_rng(3)
    T, live = 40, [40, 0, 1, 17, 33]
    parent = np.stack([W.tree_uniform(r, T)[0] for _ in range(5)])
    check(P, 9, 5, T, 16, 4, 128, 64, 6, [100, 128, 0, 735, 64], parent, live)
    # 256 rows per head in a batch: two small workgroups per CU
    T, live = 64, [64, 20, 64, 33]
    parent = np.stack([W.tree_uniform(r, T)[0] for _ in range(4)])
    check(P, 10, 4, T, 32, 8, 64, 32, 40, [2400, 100, 1500, 2000], parent, live)


def test_more_pages_than_are_staged(P):
    # one split spans more than 256 pages of 32 rows
    r = np.random.default_rng(8)
    parent = np.stack([W.tree_chain(4)[0], W.tree_uniform(r, 4)[0]])
    check(P, 8, 2, 4, 128, 128, 32, 32, 270, [8640 - 4, 8300], parent)
    parent = W.tree_uniform(r, 128)[0][None]
    check(P, 9, 1, 128, 256, 128, 32, 32, 270, [8351], parent)


def test_a_chain_continues_a_prompt(P):
    # the rows after a cached beginning, as a chain of nodes
    T = 300
    check(P, 12, 1, T, 8, 2, 64, 64, 16, [700], W.tree_chain(T)[0][None])


def test_reported(P):
    r = np.random.default_rng(1)
    parent = W.tree_chain(8)[0][None]
    kv, _, table, q = make(P, 1, 1, 8, 4, 2, 32, 32, 8, [100])
    for kv_len, change, status in (([249], None, 8), ([-1], None, 8), ([100], 11, 10), ([100], -1, 10)):
        st, t = i32([0]), table.clone()
        if change is not None:
            t[0, 2] = change
        kv.tree_attention(q, t, i32(kv_len), i32(parent), dev_status=st)
        assert st.item() == status
    parent[0, 3] = 5
    st = i32([0])
    kv.tree_attention(q, table, i32([100]), i32(parent), dev_status=st)
    assert st.item() == 7


def test_graph(P):
    r = np.random.default_rng(2)
    parent = np.stack([W.tree_uniform(r, 20)[0] for _ in range(2)])
    kv, _, table, q = make(P, 2, 2, 20, 8, 2, 64, 32, 10, [500, 333])
    n, par, st = i32([500, 333]), i32(parent), i32([0])
    shape = P.AttnShape(2, 8, 2, 128, 640, P.PTD_BF16, P.PTD_BF16, 0.0)
    ws = torch.empty(P.ptd_tree_attention_workspace_bytes(shape, 20), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kv.tree_attention(q, table, n, par, out=out, workspace=ws, dev_status=st)
    for k in range(3):
        q.copy_(torch.randn(q.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(k)))
        n.copy_(i32([500 - 30 * k, 333 - k]))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, kv.tree_attention(q, table, n, par)) and st.item() == 0


@pytest.mark.parametrize("B,T,Hq,Hkv,page,S,rows", [(1, 1, 8, 2, 64, 32, 3000), (16, 1, 8, 8, 128, 64, 700), (1, 64, 4, 2, 64, 64, 1500),
                                                    (1, 64, 8, 2, 32, 32, 9000), (3, 64, 8, 2, 128, 128, 900), (2, 200, 8, 2, 64, 32, 1100)])
def test_weights_that_need_no_rounding_give_the_bf16_outputs(P, B, T, Hq, Hkv, page, S, rows):
    # scores that are whole numbers in the exponential's domain: the weights are powers of two, and
    # nothing is left of what the two kernels do differently, bit for bit
    g = torch.Generator("cuda").manual_seed(rows)
    r = np.random.default_rng(rows)
    per = -(-rows // page)
    n = B * per + 2
    kv = P.BlockKV(n, Hkv, page, S)
    q = (torch.randint(-1, 2, (B, T, Hq, 128), generator=g, device="cuda") *
         (torch.rand((B, T, Hq, 128), generator=g, device="cuda") < 0.1)).bfloat16()
    for kind, x in enumerate((kv.k_pages, kv.v_pages)):
        e = torch.randint(-2, 3, (n, Hkv, page // S), generator=g, device="cuda")
        y = torch.randint(-7, 8, x.shape, generator=g, device="cuda") if kind == 0 else \
            torch.randn(x.shape, generator=g, device="cuda")
        y = y.unflatten(2, (-1, S)) * torch.exp2(-e.float())[..., None, None]
        x.copy_(y.to(torch.float8_e4m3fn).view(torch.uint8).flatten(2, 3))
        kv.scales[..., kind] = (127 + e).to(torch.uint8)
    kp, vp = (decode(x, kv.scales[..., i], S).to(torch.bfloat16) for i, x in enumerate((kv.k_pages, kv.v_pages)))
    table = i32(r.permutation(n)[:B * per].reshape(B, per))
    lens = i32([rows - T - 5 * b for b in range(B)])
    parent = i32(np.stack([W.tree_uniform(r, T)[0] for _ in range(B)]))
    scale = float(np.float32(1) / np.float32(1.4426950408889634))  # times log2(e), in fp32: 1
    assert np.float32(scale) * np.float32(1.4426950408889634) == 1
    for od in (torch.float32, torch.bfloat16):
        out = kv.tree_attention(q, table, lens, parent, out_dtype=od, scale=scale)
        assert torch.equal(out, P.tree_attention_paged(q, kp, vp, table, lens, parent, out_dtype=od, scale=scale))
        assert out.float().abs().amax() > 0.1
