"""Host-side checks of the serving path's entry points (no GPU needed): bad arguments
are refused before anything is launched, here and in the tensor helpers."""
import pytest
import torch

import paper_2607_10661_amd as P

FAKE = 1 << 20  # aligned non-null address; every call below fails validation first


def _err(fn, *a, **kw):
    with pytest.raises(P.PTDError) as e:
        fn(*a, stream=0, **kw)
    return e.value.status


def test_status_strings_of_the_new_codes():
    for code in (12, 13, 14):
        assert P.ptd_status_string(code) != "unknown status" and code in P.STATUS
    assert P.ptd_status_string(15) == "unknown status"


def _prompt(B=2, N=100, Hq=8, Hkv=2, D=128, ldq=0, ldk=0, ldv=0, dt=P.PTD_BF16, od=P.PTD_BF16, scale=0.0):
    return P.PromptShape(B, N, Hq, Hkv, D, ldq, ldk, ldv, dt, od, scale)


def test_prompt_attention_refusals():
    A = P.ptd_prompt_attention
    ok = (FAKE, FAKE, FAKE, FAKE, FAKE)
    for i in range(5):
        assert _err(A, *[None if j == i else x for j, x in enumerate(ok)], _prompt()) == 1
    for bad in (dict(B=0), dict(B=65537), dict(N=-1), dict(Hq=0), dict(Hkv=0), dict(Hq=7), dict(D=96), dict(D=32),
                dict(ldq=8 * 128 - 8), dict(ldk=2 * 128 - 8), dict(ldv=128), dict(N=2 ** 30, Hq=8),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(ldq=-1024)):
        assert _err(A, *ok, _prompt(**bad)) == 2, bad
    assert _err(A, *ok, _prompt(dt=2)) == 3
    assert _err(A, *ok, _prompt(od=7)) == 3
    for i in (0, 1, 2, 4):
        assert _err(A, *[x + 8 if j == i else x for j, x in enumerate(ok)], _prompt()) == 4
    assert _err(A, *ok, _prompt(ldq=1024 + 4)) == 4
    assert _err(A, *ok, _prompt(ldk=256 + 2, dt=P.PTD_F32)) == 4
    P.ptd_prompt_attention(None, None, None, FAKE, None, _prompt(N=0), stream=0)  # nothing to do


def _state(B=2, page=64, per=8, num=16, **kw):
    s = P.PageState(FAKE, FAKE, FAKE, FAKE, B, page, per, num)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def test_page_plan_refusals():
    for f in ("page_table", "num_held", "free_pages", "num_free"):
        assert _err(P.ptd_page_init, _state(**{f: None})) == 1
        assert _err(P.ptd_page_plan, _state(**{f: None}), FAKE, FAKE, 10, 0, FAKE, FAKE) == 1
    for bad in (dict(B=0), dict(B=65537), dict(page=0), dict(page=48), dict(page=1 << 21), dict(per=0), dict(num=0),
                dict(per=1 << 26), dict(num=1 << 25)):
        assert _err(P.ptd_page_init, _state(**bad)) == 2, bad
        assert _err(P.ptd_page_plan, _state(**bad), FAKE, FAKE, 10, 0, FAKE, FAKE) == 2, bad
    A = P.ptd_page_plan
    assert _err(A, _state(), None, FAKE, 10, 0, FAKE, FAKE) == 1
    assert _err(A, _state(), FAKE, None, 10, 0, FAKE, FAKE) == 1
    assert _err(A, _state(), FAKE, FAKE, 10, 0, None, FAKE) == 1       # packed rows need their starts
    assert _err(A, _state(), FAKE, FAKE, 10, 0, FAKE, None) == 1
    assert _err(A, _state(), FAKE, FAKE, -1, 0, FAKE, FAKE) == 2
    assert _err(A, _state(), FAKE, FAKE, 10, -1, FAKE, FAKE) == 2
    assert _err(A, _state(), FAKE, FAKE, 10, 4, None, FAKE) == 2       # N != B * rows_per_seq


def _blocks(page=64, per=32, num=64, S=32, **kw):
    s = P.KVPagesFp8Blk(FAKE, FAKE, FAKE, FAKE, page, per, num, S)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def test_write_refusals():
    def w(k=FAKE, v=FAKE, dt=P.PTD_BF16, ldk=256, ldv=256, N=10, slots=FAKE, src=None, rows=0, kv=None, Hkv=2, D=128):
        return _err(P.ptd_kv_write_fp8blk, k, v, dt, ldk, ldv, N, slots, src, rows, kv or _blocks(), Hkv, D)

    assert w(k=None) == 1 and w(v=None) == 1 and w(slots=None) == 1
    for f in ("k_pages", "v_pages", "scales"):
        assert w(kv=_blocks(**{f: None})) == 1
    assert w(dt=5) == 3
    for bad in (dict(page=48), dict(page=16), dict(num=0), dict(S=16), dict(S=48), dict(S=256), dict(page=32, S=64),
                dict(num=1 << 25)):
        assert w(kv=_blocks(**bad)) == 2, bad
    for bad in (dict(N=-1), dict(Hkv=0), dict(D=64), dict(ldk=248), dict(ldv=128), dict(src=FAKE), dict(src=FAKE, rows=3),
                dict(src=FAKE, rows=-2)):
        assert w(**bad) == 2, bad
    for bad in (dict(k=FAKE + 8), dict(v=FAKE + 2), dict(ldk=260), dict(kv=_blocks(k_pages=FAKE + 8)),
                dict(kv=_blocks(v_pages=FAKE + 4)), dict(kv=_blocks(scales=FAKE + 2)), dict(dt=P.PTD_F32, ldv=258)):
        assert w(**bad) == 4, bad
    P.ptd_kv_write_fp8blk(None, None, P.PTD_BF16, 256, 256, 0, None, None, 0, _blocks(), 2, 128, stream=0)


def test_block_attention_refusals():
    def shape(Hq=8, Hkv=2, D=128, L=2048, dt=P.PTD_BF16, od=P.PTD_BF16):
        return P.AttnShape(1, Hq, Hkv, D, L, dt, od, 0.0)

    def a(kv=None, s=None, q=FAKE, T=64, **kw):
        return _err(P.ptd_tree_attention_paged_fp8blk, q, kv or _blocks(), FAKE, None, FAKE, T, FAKE, s or shape(), **kw)

    for f in ("k_pages", "v_pages", "scales", "page_table"):
        assert a(kv=_blocks(**{f: None})) == 1
    assert a(q=None) == 1
    assert a(s=shape(dt=P.PTD_F32, od=P.PTD_F32)) == 3
    for bad in (dict(page=48), dict(page=16), dict(per=31), dict(num=0), dict(S=16), dict(S=128), dict(S=0)):
        assert a(kv=_blocks(**bad)) == 2, bad
    assert a(s=shape(D=64)) == 2 and a(s=shape(Hq=7)) == 2 and a(T=0) == 2
    assert a(kv=_blocks(scales=FAKE + 2)) == 4 and a(kv=_blocks(v_pages=FAKE + 8)) == 4
    assert a() == 5 and a(workspace=FAKE, workspace_bytes=16) == 5


def test_helpers_refuse_what_the_calls_cannot_see():
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # host tensors
        P.prompt_attention(x, x, x, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        P.BlockKV(4, 2, 64, 48, device="cpu")
    wide = torch.zeros((4, 6, 64), dtype=torch.bfloat16)
    assert P._rows(x) == 128 and P._rows(wide[:, 1:3]) == 384 and P._rows(x[:1]) == 128
    for bad in (x[:1].expand(4, 2, 64), x.transpose(0, 1), wide[:, ::2], wide[..., ::2], x[0]):
        with pytest.raises(ValueError):  # a stride of 0 would stand for dense rows
            P._rows(bad)
    with pytest.raises(ValueError):
        P.BlockKV(4, 2, 32, 64, device="cpu")
    kv = P.BlockKV(4, 2, 64, 32, device="cpu")
    with pytest.raises(ValueError):
        kv.write(torch.zeros((4, 2, 128), dtype=torch.bfloat16), torch.zeros((4, 2, 128), dtype=torch.bfloat16),
                 torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        P.PageTables(2, 64, 4, 8, device="cpu")


def test_block_attention_helper_counts_what_the_kernel_reads(monkeypatch):
    # tensors on the host, as if they were on the GPU: a helper that lets one through reaches the call
    monkeypatch.setattr(P, "_need_gpu", lambda *ts: None)
    monkeypatch.setattr(P, "_need_here", lambda *ts: None)
    monkeypatch.setattr(P, "ptd_tree_attention_paged_fp8blk", lambda *a: reached.append(a))
    reached = []
    kv = P.BlockKV(4, 2, 64, 32, device="cpu")
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)
    good = dict(q=torch.zeros((2, 8, 4, 128), dtype=torch.bfloat16), page_table=i32(2, 2), kv_len=i32(2), parent=i32(2, 8))
    kv.tree_attention(**good, tree_len=i32(2))
    assert len(reached) == 1
    for bad in (dict(tree_len=i32(1)), dict(tree_len=i32(3)), dict(kv_len=i32(1)), dict(page_table=i32(4)),
                dict(page_table=i32(1, 4)), dict(parent=i32(2, 7)), dict(parent=i32(16)),
                dict(workspace=torch.zeros(1, dtype=torch.uint8).expand(1 << 24))):
        with pytest.raises(ValueError):
            kv.tree_attention(**dict(good, **bad))
    assert len(reached) == 1
