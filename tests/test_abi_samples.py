"""Host-side checks of the entry points for several samples of one prompt (no GPU needed): bad
arguments are refused before anything is launched, here and in the tensor helpers."""
import math

import pytest
import torch

import paper_2607_10661_amd as P

FAKE = 1 << 20  # aligned non-null address; every call below fails validation first


def _err(fn, *a, **kw):
    with pytest.raises(P.PTDError) as e:
        fn(*a, stream=0, **kw)
    return e.value.status


def _qk(**kw):
    d = dict(N=10, Hq=8, Hkv=2, D=128, rot_dim=128, pairing=0, norm=1, dtype=P.PTD_BF16, w_dtype=P.PTD_BF16, ldq=0, ldk=0, ldv=0,
             ldqo=0, ldko=0, eps=1e-6, theta=10000.0)
    d.update(kw)
    return P.QKShape(*d.values())


def test_qk_norm_rope_refusals():
    def a(shape=None, q=FAKE, k=FAKE, v=None, wq=FAKE, wk=FAKE, pos=FAKE, slots=None, qo=FAKE, ko=FAKE, store=None, inv=None):
        return _err(P.ptd_qk_norm_rope, q, k, v, wq, wk, pos, slots, qo, ko, store, shape or _qk(), inv)

    assert a(q=None) == a(k=None) == a(pos=None) == a(qo=None) == a(ko=None) == 1
    for bad in (dict(N=-1), dict(N=(1 << 26) - 3), dict(Hq=-1), dict(Hkv=-1), dict(Hq=0, Hkv=0), dict(Hq=65536), dict(D=96), dict(D=256), dict(rot_dim=-16),
                dict(rot_dim=144), dict(rot_dim=8), dict(rot_dim=72), dict(D=64), dict(pairing=2), dict(pairing=-1), dict(norm=2),
                dict(norm=-1), dict(norm=0), dict(eps=-1e-6), dict(eps=math.nan), dict(eps=math.inf), dict(theta=0.0), dict(theta=-1.0),
                dict(theta=math.inf), dict(theta=math.nan), dict(ldq=1016), dict(ldk=248), dict(ldv=128), dict(ldqo=-1024), dict(ldko=8)):
        assert a(_qk(**bad)) == 2, bad
    for f in (math.nan, math.inf, 2.0 ** 21):
        assert a(inv=[1.0] * 63 + [f]) == 2
    assert a(_qk(dtype=2)) == 3 and a(_qk(w_dtype=-1)) == 3
    for bad in (dict(q=FAKE + 8), dict(k=FAKE + 2), dict(wq=FAKE + 4), dict(wk=FAKE + 8), dict(qo=FAKE + 4), dict(ko=FAKE + 8)):
        assert a(**bad) == 4, bad
    assert a(_qk(ldq=1028)) == 4 and a(_qk(ldko=258)) == 4 and a(_qk(dtype=P.PTD_F32, ldk=258)) == 4
    with pytest.raises(ValueError):
        P.ptd_qk_norm_rope(FAKE, FAKE, None, None, None, FAKE, None, FAKE, FAKE, None, _qk(), [1.0] * 63, stream=0)
    store = lambda *x: P.KVStore(*x)  # noqa: E731
    ok = dict(v=FAKE, slots=FAKE)
    assert a(store=store(None, FAKE, 64, 4), **ok) == 1 and a(store=store(FAKE, None, 64, 4), **ok) == 1
    assert a(store=store(FAKE, FAKE, 64, 4), v=FAKE) == 1 and a(store=store(FAKE, FAKE, 64, 4), slots=FAKE) == 1
    for bad in ((0, 4), (64, 0), (1 << 20, 1 << 11)):
        assert a(store=store(FAKE, FAKE, *bad), **ok) == 2
    assert a(_qk(Hkv=0), k=None, ko=None, wk=None, store=store(FAKE, FAKE, 64, 4), **ok) == 2
    assert a(store=store(FAKE + 8, FAKE, 64, 4), **ok) == 4 and a(store=store(FAKE, FAKE + 2, 64, 4), **ok) == 4
    assert a(store=store(FAKE, FAKE, 64, 4), v=FAKE + 8, slots=FAKE) == 4
    P.ptd_qk_norm_rope(None, None, None, None, None, None, None, None, None, None, _qk(N=0), stream=0)  # nothing to do


def test_token_logprobs_refusals():
    def a(x=FAKE, dt=P.PTD_BF16, R=10, V=1000, ld=1000, tok=FAKE, nodes=None, T=0, tau=1.0, k=4, lp=FAKE, ent=FAKE, idx=FAKE,
          val=FAKE, ws=None, n=0):
        return _err(P.ptd_token_logprobs, x, dt, R, V, ld, tok, nodes, T, tau, k, lp, ent, idx, val, ws, n)

    assert a(x=None) == 1 and a(tok=None) == 1 and a(tok=None, lp=None, nodes=FAKE, T=4) == 1
    assert a(k=0, lp=None, ent=None, idx=None, val=None) == 1
    assert a(dt=2) == 3
    for bad in (dict(R=0), dict(R=-1), dict(R=1 << 24), dict(R=1 << 20, V=262144, ld=262144, dt=P.PTD_F32), dict(V=0), dict(V=262145, ld=262145), dict(ld=999), dict(k=-1), dict(k=17), dict(V=3, ld=3), dict(k=0),
                dict(idx=None, val=None), dict(tau=0.0), dict(tau=-1.0), dict(tau=math.nan), dict(tau=math.inf), dict(tau=1e-31), dict(tau=1e31),
                dict(nodes=FAKE, T=0), dict(nodes=FAKE, T=3), dict(nodes=FAKE, T=1025)):
        assert a(**bad) == 2, bad
    assert a(x=FAKE + 1) == 4 and a(x=FAKE + 2, dt=P.PTD_F32) == 4
    big = dict(V=128256, ld=128256)
    need = P.ptd_token_logprobs_workspace_bytes(10, 128256, 4)
    assert need > 0
    assert a(**big) == 5 and a(**big, ws=FAKE, n=16) == 5 and a(**big, ws=FAKE + 4, n=need) == 4
    assert P.ptd_token_logprobs_workspace_bytes(10, 1000, 4) == 0
    assert P.ptd_token_logprobs_workspace_bytes(3 << 20, 32768, 4) == (3 << 20) * 2 * (32 + 8 * 16)  # fp32: two slices
    assert P.ptd_token_logprobs_workspace_bytes((1 << 24) - 1, 16384, 4) == 0 and P.ptd_token_logprobs_workspace_bytes((1 << 20) - 1, 262144, 16) > 0
    for bad in ((0, 1000, 4), (10, 0, 0), (10, 262145, 4), (10, 1000, 17), (10, 3, 4), (10, 1000, -1)):
        assert P.ptd_token_logprobs_workspace_bytes(*bad) == 0


def _state(B=2, page=64, per=8, num=16, **kw):
    s = P.PageState(FAKE, FAKE, FAKE, FAKE, B, page, per, num)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


BAD_STATES = (dict(B=0), dict(B=65537), dict(page=0), dict(page=48), dict(page=1 << 21), dict(per=0), dict(num=0), dict(per=1 << 26),
              dict(num=1 << 25))


def test_shared_page_refusals():
    plan = lambda s, *a: _err(P.ptd_page_plan_shared, s, *a)  # noqa: E731
    ok = (FAKE, FAKE, FAKE, 10, 0, FAKE, FAKE)
    fork = (FAKE,) * 8
    out = 2 * FAKE
    for f in ("page_table", "num_held", "free_pages", "num_free"):
        assert plan(_state(**{f: None}), *ok) == 1
        assert _err(P.ptd_page_fork, _state(**{f: None}), *fork) == 1
        assert _err(P.ptd_page_compact, _state(**{f: None}), FAKE, FAKE, FAKE) == 1
    for bad in BAD_STATES:
        assert plan(_state(**bad), *ok) == 2
        assert _err(P.ptd_page_fork, _state(**bad), *fork) == 2
        assert _err(P.ptd_page_compact, _state(**bad), FAKE, FAKE, FAKE) == 2
    for i in (0, 1, 2, 5, 6):
        assert plan(_state(), *[None if j == i else x for j, x in enumerate(ok)]) == 1
    assert plan(_state(), FAKE, FAKE, FAKE, -1, 0, FAKE, FAKE) == 2 and plan(_state(), FAKE, FAKE, FAKE, 10, 4, None, FAKE) == 2
    good = (FAKE, FAKE, FAKE, out, out, FAKE, FAKE, FAKE)
    for i in range(8):
        assert _err(P.ptd_page_fork, _state(), *[None if j == i else x for j, x in enumerate(good)]) == 1
    assert _err(P.ptd_page_fork, _state(), FAKE, FAKE, FAKE, FAKE, out, FAKE, FAKE, FAKE) == 2  # the state's own table
    assert _err(P.ptd_page_fork, _state(), FAKE, FAKE, FAKE, out, FAKE, FAKE, FAKE, FAKE) == 2
    for i in range(3):
        assert _err(P.ptd_page_compact, _state(), *[None if j == i else FAKE for j in range(3)]) == 1


def test_page_copy_refusals():
    def a(arrays=None, pages=8, n=4, src=FAKE, dst=FAKE, rows=None):
        return _err(P.ptd_page_copy, [P.PageArray(FAKE, 2, 64, 1, 256)] if arrays is None else arrays, pages, n, src, dst, rows)

    assert a(src=None) == 1 and a(dst=None) == 1 and a([P.PageArray(None, 2, 64, 1, 256)]) == 1
    assert a(pages=0) == 2 and a(n=-1) == 2
    for bad in ((0, 64, 1, 256), (2, 0, 1, 256), (2, 64, 0, 256), (2, 64, 1, 0), (1 << 10, 1 << 10, 1, 1 << 11), (1, 1 << 16, 1, 1 << 16)):
        assert a([P.PageArray(FAKE, 2, 64, 1, 256), P.PageArray(FAKE, *bad)]) == 2, bad
    P.ptd_page_copy([], 8, 4, FAKE, FAKE, stream=0)  # nothing to do
    P.ptd_page_copy([P.PageArray(FAKE, 2, 64, 1, 256)], 8, 0, None, None, stream=0)


def test_helpers_refuse_what_the_calls_cannot_see(monkeypatch):
    # tensors on the host, as if they were on the GPU: a helper that lets one through reaches the call
    x = torch.zeros((4, 6, 128), dtype=torch.bfloat16)
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):  # host tensors
        P.qk_norm_rope(x, x, i32(4))
    with pytest.raises(ValueError):
        P.token_logprobs(torch.zeros((2, 10)), i32(2))
    monkeypatch.setattr(P, "_need_here", lambda *ts: None)
    reached = []
    monkeypatch.setattr(P, "ptd_qk_norm_rope", lambda *a: reached.append(a))
    monkeypatch.setattr(P, "ptd_token_logprobs", lambda *a: reached.append(a))
    q, k, v = x[:, :4], x[:, 4:5], x[:, 5:]
    pages = torch.zeros((3, 1, 32, 128), dtype=torch.bfloat16)
    good = dict(q=q, k=k, positions=i32(4), v=v, slots=i32(4), k_pages=pages, v_pages=pages.clone())
    P.qk_norm_rope(**good)
    assert len(reached) == 1
    w = torch.ones(128)
    for bad in (dict(k=k[:3]), dict(k=k.float()), dict(k=k[..., :64]), dict(positions=i32(3)), dict(positions=i32(4).long()), dict(slots=i32(5)),
                dict(slots=None), dict(v=None), dict(v=v[:3]), dict(k_pages=None), dict(v_pages=pages[:2]), dict(k_pages=pages.float()),
                dict(k_pages=pages[:, :, ::2], v_pages=pages[:, :, ::2]), dict(q_weight=w[:64]), dict(q_weight=w, k_weight=w.bfloat16()),
                dict(eps=None, q_weight=w), dict(q_out=torch.zeros((4, 4, 128))), dict(k_out=torch.zeros((3, 1, 128), dtype=torch.bfloat16)),
                dict(q=x[:1].expand(4, 6, 128)), dict(q=x[:, ::2]), dict(k_pages=pages[:, 0], v_pages=pages[:, 0])):
        with pytest.raises(ValueError):
            P.qk_norm_rope(**dict(good, **bad))
    y = torch.zeros((6, 10))
    good = dict(logits=y, tokens=i32(6))
    P.token_logprobs(**good)
    P.token_logprobs(y.view(2, 3, 10), i32(2, 3), nodes=i32(2, 2))
    assert len(reached) == 3
    for bad in (dict(tokens=i32(5)), dict(tokens=i32(6).long()), dict(nodes=i32(2, 3)), dict(nodes=i32(6)), dict(tokens=None, nodes=i32(2, 2)),
                dict(logits=y.t()), dict(logits=y[:1].expand(6, 10)), dict(workspace=torch.zeros(1, dtype=torch.uint8).expand(1 << 20))):
        with pytest.raises(ValueError):
            P.token_logprobs(**dict(good, **bad))
    assert len(reached) == 3
