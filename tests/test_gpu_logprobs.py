"""GPU checks of ptd_token_logprobs against a plain 64-bit implementation; tolerances are the
error bounds that ref64_samples.logprobs works out per row."""
import math
import random

import numpy as np
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
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32).cuda()


def logits(R_, V, dtype, seed, odd=0, std=2.0, peak=0.0, masked=0.0):
    g = torch.Generator("cuda").manual_seed(seed)
    x = (torch.randn((R_, V + odd), generator=g, device="cuda") * std).to(dtype)[:, :V]
    if peak:
        at = torch.randint(V, (R_, 1), generator=g, device="cuda")
        x.scatter_(1, at, (torch.rand((R_, 1), generator=g, device="cuda") * peak).to(dtype))
    if masked:
        drop = torch.rand((R_, V), generator=g, device="cuda") < masked
        x.masked_fill_(drop, -math.inf)
    return x


def check(got, x, tokens, k, tau=1.0, rows=None):
    lp, ent, idx, val = [None if t is None else t.double().cpu() for t in got]
    x = x.cpu()
    for r in range(x.shape[0] if tokens is None else len(tokens)):
        t = None if tokens is None else tokens[r]
        at = r if rows is None else rows[r]
        if t is not None and t < 0:
            assert lp[r] == 0 and (ent is None or ent[r] == 0)
            assert not k or ((idx[r] == -1).all() and (val[r] == 0).all())
            continue
        w_lp, w_ent, order, top, e_lp, e_ent = R.logprobs(x[at], tau, t, k)
        if t is not None:
            assert lp[r] == w_lp or abs(lp[r] - w_lp) <= e_lp + 2.0 ** -24 * abs(w_lp), (r, lp[r], w_lp, e_lp)
        if ent is not None:
            assert abs(ent[r] - w_ent) <= e_ent, (r, ent[r], w_ent, e_ent)
        if k:
            assert idx[r].int().tolist() == order, (r, idx[r].tolist(), order)
            for a, b in zip(val[r].tolist(), top):
                assert a == b or abs(a - b) <= e_lp + 2.0 ** -24 * abs(b), (r, a, b, e_lp)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1, 2, 7, 17, 129, 1000, 4096, 4099, 16384, 32003, 65541, 128256])
def test_rows(P, dtype, V):
    for n, (N, k, tau, odd) in enumerate([(1, min(16, V), 1.0, 0), (5, min(3, V), 0.7, 1), (9, 0, 2.0, 3), (3, min(8, V), 1.0, 0)]):
        if V > 40000:
            N = min(N, 3)
        x = logits(N, V, dtype, n, odd, std=[2.0, 0.01, 6.0, 2.0][n], peak=[0, 24, 0, 40][n])
        r = random.Random(V + n)
        tok = [r.choice([x[i].argmax().item(), r.randrange(V)]) for i in range(N)]
        st = i32([0])
        check(P.token_logprobs(x, i32(tok), k, temperature=tau, dev_status=st), x, tok, k, tau)
        assert st.item() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,N", [(50, 700), (3000, 300), (20000, 260), (70000, 130)])
def test_many_rows(P, dtype, V, N):
    # one slice and several per row, few and many rows
    x = logits(N, V, dtype, V, peak=20)
    tok = [i % V for i in range(N)]
    tok[1] = tok[N - 1] = -1
    got = P.token_logprobs(x, i32(tok), 5)
    some = [0, 1, 2, N // 2, N - 2, N - 1]
    check([t[some] for t in got], x[some], [tok[i] for i in some], 5)


@pytest.mark.parametrize("V", [300, 40000])
def test_decided_rows_keep_their_precision(P, V):
    # one entry with all but 1e-4 .. 1e-30 of the mass: log probability and entropy are next to 0
    x = torch.zeros((6, V), device="cuda")
    for i, top in enumerate((20.0, 30.0, 40.0, 60.0, 80.0, 100.0)):
        x[i, 7 * i] = top
    tok = [7 * i for i in range(6)]
    lp, ent, _, _ = P.token_logprobs(x, i32(tok))
    for i, top in enumerate((20.0, 30.0, 40.0, 60.0, 80.0, 100.0)):
        rest = (V - 1) * math.exp(-top)
        # V terms of one value, 71 roundings and the argument's: 3 * 2^-24 * top
        rel = 2.0 ** -24 * (80 + 4 * top)
        if rest < 1e-38:
            assert -1e-38 <= lp[i].item() <= 0
            continue
        assert abs(lp[i].item() + math.log1p(rest)) <= rel * rest
        want = math.log1p(rest) + rest * top / (1 + rest)
        assert abs(ent[i].item() - want) <= 2 * rel * want
    # two entries that share the mass
    x[:, 5] = 100.0
    x[:, 11] = 100.0
    lp, ent, idx, val = P.token_logprobs(x[:4], i32([5, 11, 5, 11]), 2)
    assert (lp + math.log(2)).abs().max() <= 1e-7 and (ent - math.log(2)).abs().max() <= 1e-7
    assert idx.tolist() == [[5, 11]] * 4 and torch.equal(val[:, 0], lp)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [64, 20000, 100000])
def test_masked_entries(P, dtype, V):
    x = logits(4, V, dtype, 3, masked=0.9)
    x[1, 1:] = -math.inf            # one entry left
    x[1, 0] = 3.0
    x[2] = -math.inf                # nothing left
    x[3, : V // 2] = -math.inf      # whole slices without an entry
    x[3, V - 1] = 1.0
    tok = [x[0].argmax().item(), 0, 5, 0]
    k = min(16, V)
    got = P.token_logprobs(x, i32(tok), k)
    check(got, x, tok, k)
    assert got[0][1] == 0 and got[1][1] == 0 and got[0][2] == -math.inf and got[0][3] == -math.inf and got[1][2] == 0
    assert got[2][2].tolist() == list(range(k)) and (got[3][2] == -math.inf).all()
    # fewer entries than k: the masked ones follow by index
    assert got[2][1].tolist() == list(range(k)) and (got[3][1][1:] == -math.inf).all()
    lowest = torch.full((1, V), torch.finfo(dtype).min, dtype=dtype, device="cuda")  # a mask of the type's lowest value
    lowest[0, 3] = 0.5
    check(P.token_logprobs(lowest, i32([3]), 4), lowest, [3], 4)
    lowest[0, 3] = torch.finfo(dtype).min  # all at the lowest value: uniform
    lp, ent, _, _ = P.token_logprobs(lowest, i32([3]))
    assert abs(lp.item() + math.log(V)) <= 1e-6 * math.log(V) and abs(ent.item() - math.log(V)) <= 1e-6 * math.log(V)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [100, 50000])
def test_not_numbers_stay_in_their_row(P, dtype, V):
    x = logits(6, V, dtype, 5)
    want = P.token_logprobs(x, i32([3] * 6), 4)
    x[1, 50], x[3, 7], x[4, V - 1] = float("nan"), float("inf"), -float("nan")
    lp, ent, idx, val = P.token_logprobs(x, i32([3] * 6), 4)
    for got, w in zip((lp, ent, idx, val), want):
        assert torch.equal(got[[0, 2, 5]], w[[0, 2, 5]])
    assert lp[[1, 3, 4]].isnan().all() and ent[[1, 3, 4]].isnan().all()
    assert ((idx >= -1) & (idx < V)).all()


def test_ties_and_signed_zeros(P):
    for dtype in (torch.bfloat16, torch.float32):
        for V in (40, 40000):
            x = torch.zeros((3, V), dtype=dtype, device="cuda")
            x[0, ::2] = -0.0
            x[1, 7::3] = 1.0
            x[2] = -5.0
            x[2, V - 1] = -4.0
            check(P.token_logprobs(x, i32([1, 7, 0]), 16), x, [1, 7, 0], 16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,N", [(1000, 1), (40000, 1), (40000, 300)])
def test_rows_in_order(P, dtype, V, N):
    # ascending and descending rows: the reference moves with every group of chunks, candidates fill their lists
    up = torch.linspace(-90, 90, V, device="cuda").to(dtype)
    steep = torch.linspace(-3000, 3000, V, device="cuda").to(dtype)
    x = torch.stack([up, up.flip(0), steep, steep.flip(0)] * N)
    tok = [V - 1, 0, V - 2, 3] * N
    got = P.token_logprobs(x, i32(tok), 16)
    check([t[:4] for t in got], x[:4], tok[:4], 16)
    for t in got:
        assert torch.equal(t.view(N, -1), t.view(N, -1)[:1].expand(N, -1))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,N,k,odd", [(1, 600, 1, 0), (3, 600, 2, 1), (17, 1100, 16, 3), (50, 5000, 5, 0), (129, 700, 0, 1), (500, 520, 4, 5),
                                       (511, 1030, 16, 1), (1024, 513, 8, 0), (1025, 2050, 3, 1), (2041, 4100, 9, 7), (2048, 2048, 5, 0),
                                       (4096, 2048, 5, 0), (4091, 8200, 0, 0)])
def test_many_short_rows(P, dtype, V, N, k, odd):
    x = logits(N, V, dtype, V + N, odd=odd, peak=20.0, masked=0.2)
    x[3] = -math.inf                               # nothing left
    x[4] = 2.0                                     # ties
    x[5, V // 2] = float("nan")
    x[6, 0] = float("inf")
    x[7] = torch.finfo(dtype).min                  # the type's lowest value throughout
    x[8, ::2] = -0.0
    x[8, 1::2] = 0.0
    x[9] = torch.linspace(-50, 50, V).to(dtype)
    x[10] = x[9].flip(0)
    tok = torch.randint(0, V, (N,), generator=torch.Generator().manual_seed(V)).tolist()
    tok[11] = -1
    st = i32([0])
    got = P.token_logprobs(x, i32(tok), k, dev_status=st)
    assert st.item() == 0
    some = [0, 1, 2, 3, 4, 7, 8, 9, 10, 11] + list(range(N - 30, N))
    check([None if t is None else t[some] for t in got], x[some], [tok[r] for r in some], k)
    assert got[0][5:7].isnan().all() and got[1][5:7].isnan().all()
    # the workgroups' kernel, a few rows at a time
    near = P.token_logprobs(x[100:200], i32(tok[100:200]), k)
    if k:
        assert torch.equal(near[2], got[2][100:200])
    live = near[0] > -math.inf
    assert torch.equal(live, got[0][100:200] > -math.inf)
    assert ((near[0] - got[0][100:200])[live].abs() <= 2e-5 * (1 + near[0][live].abs())).all()


def test_many_short_rows_along_paths(P):
    B, T, V = 40, 64, 300
    r = random.Random(5)
    x = logits(B * (T + 1), V, torch.bfloat16, 9)
    paths = [sorted(r.sample(range(T), r.choice([0, 1, 3, 9]))) for _ in range(B)]
    tok, rows = [], []
    for b, p in enumerate(paths):
        tok += [r.randrange(V) if j <= len(p) else -1 for j in range(T + 1)]
        rows += [b * (T + 1) + (p[j - 1] + 1 if 0 < j <= len(p) else 0) for j in range(T + 1)]
    nodes = i32([p + [-1] * (T - len(p)) for p in paths])
    st = i32([0])
    check(P.token_logprobs(x, i32(tok), 5, nodes=nodes, dev_status=st), x, tok, 5, rows=rows)
    assert st.item() == 0
    tok[0], tok[T + 2] = V, 5
    nodes[1, 0] = T
    got = P.token_logprobs(x, i32(tok), 5, nodes=nodes, dev_status=st)
    assert st.item() in (13, 14) and got[0][0] == 0 and got[0][T + 2] == 0 and (got[2][0] == -1).all()


@pytest.mark.parametrize("tau", [1e-3, 0.05, 10.0, 1e6])
def test_temperatures(P, tau):
    x = logits(3, 5000, torch.float32, 8, peak=10)
    tok = [x[0].argmax().item(), 9, x[2].argmax().item()]
    check(P.token_logprobs(x, i32(tok), 6, temperature=tau), x, tok, 6, tau)


@pytest.mark.parametrize("B,T,V", [(1, 1, 33), (3, 16, 1000), (16, 64, 4003), (2, 5, 70000), (5, 300, 129)])
def test_paths(P, B, T, V):
    r = random.Random(T)
    x = logits(B * (T + 1), V, torch.bfloat16, 11, peak=10).view(B, T + 1, V)
    paths = [sorted(r.sample(range(T), r.randint(0, min(T, 6)))) for _ in range(B)]
    nodes = [p + [-1] * (T - len(p)) for p in paths]
    tokens = [[r.randrange(V) if j <= len(p) else -1 for j in range(T + 1)] for p in paths]
    rows = [b * (T + 1) + (0 if j == 0 or j > len(p) else p[j - 1] + 1) for b, p in enumerate(paths) for j in range(T + 1)]
    st = i32([0])
    got = P.token_logprobs(x, i32(tokens), 3, nodes=i32(nodes), dev_status=st)
    check(got, x.view(-1, V), [t for row in tokens for t in row], 3, rows=rows)
    assert st.item() == 0


def test_paths_of_verify(P):
    # the outputs of verify as they are: the log probability of every emitted token
    import workloads as W
    w = W.make_workload("tiny")
    x = torch.from_numpy(w.logits).cuda()
    V = x.shape[-1]
    x = x.view(-1, V)
    am, _, _ = P.topk_argmax(x, 1)
    al, an, ot = P.verify(am.view(w.B, w.T + 1), i32(w.tokens), i32(w.parent))
    lp, ent, _, _ = P.token_logprobs(x, ot.view(-1), nodes=an)
    n = al.item()
    assert n == w.planted_depth[0] and n > 0
    at = 0
    for j in range(n + 1):
        ref = torch.log_softmax(x[at].double(), 0)
        assert abs(lp[j].item() - ref[ot[0, j].long()].item()) <= 1e-5
        assert ref.argmax() == ot[0, j]
        at = an[0, j].item() + 1 if j < n else at
    assert (lp[n + 1:] == 0).all() and (ent[n + 1:] == 0).all()


def test_reported_entries(P):
    V = 500
    x = logits(8, V, torch.float32, 2)
    for bad in (V, 2 ** 31 - 1, -2):
        st = i32([0])
        tok = [3, bad, 5, -1, 0, V - 1, 7, 8]
        check(P.token_logprobs(x, i32(tok), 2, dev_status=st), x, [t if 0 <= t < V else -1 for t in tok], 2)
        assert st.item() == 14
    for bad in (3, -1, 2 ** 31 - 1, -2 ** 31):
        st = i32([0])
        got = P.token_logprobs(x, i32([1, 2, 3, -1, 4, 5, -1, -1]), 2, nodes=i32([[0, bad, 2], [1, 0, 0]]), dev_status=st)
        check(got, x, [1, 2, -1, -1, 4, 5, -1, -1], 2, rows=[0, 1, 0, 0, 4, 6, 0, 0])
        assert st.item() == 13


def test_some_outputs(P):
    x = logits(4, 30000, torch.bfloat16, 6)
    lp, ent, idx, val = P.token_logprobs(x, i32([1, 2, 3, 4]), 4)
    a = P.token_logprobs(x, None, 4)
    assert a[0] is None and torch.equal(a[1], ent) and torch.equal(a[2], idx) and torch.equal(a[3], val)
    b = P.token_logprobs(x, i32([1, 2, 3, 4]), 0, with_entropy=False)
    assert torch.equal(b[0], lp) and b[1] is None and b[2] is None
    am, ti, tv = P.topk_argmax(x, 4)
    assert torch.equal(ti, idx)
    only = torch.empty((4, 4), dtype=torch.float32, device="cuda")
    ws = torch.empty(P.ptd_token_logprobs_workspace_bytes(4, 30000, 4) + 1, dtype=torch.uint8, device="cuda")
    P.ptd_token_logprobs(x, P.PTD_BF16, 4, 30000, 30000, None, None, 0, 1.0, 4, None, None, None, only, ws, ws.numel())
    assert torch.equal(only, val)


def test_graph_streams_and_two_calls(P):
    x = logits(6, 50000, torch.bfloat16, 1)
    tok = i32([1, 2, 3, 4, 5, -1])
    ws = torch.empty(P.ptd_token_logprobs_workspace_bytes(6, 50000, 8), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = P.token_logprobs(x, tok, 8, workspace=ws)
    for r in range(4):
        x.copy_(logits(6, 50000, torch.bfloat16, 20 + r))
        tok.copy_(torch.tensor([r, 7, -1, 9, 49999, 3]))
        g.replay()
        torch.cuda.synchronize()
        eager = P.token_logprobs(x, tok, 8, workspace=ws)  # the same workspace, in order
        for a, b in zip(out, eager):
            assert torch.equal(a, b)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(P.token_logprobs(x, tok, 8))
    torch.cuda.synchronize()
    for y in got:
        for a, b in zip(y, eager):
            assert torch.equal(a, b)


def test_rows_past_32_bits(P):
    # rows whose elements start past 2^31: 20000 rows of 131072 bf16, a few of them read
    N, V = 17000, 131072
    x = torch.zeros((N, V), dtype=torch.bfloat16, device="cuda")
    tok = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    at = [0, 16390, N - 1]
    for i, r in enumerate(at):
        x[r, 1000 + i] = 5.0
        tok[r] = 1000 + i
    lp, ent, idx, _ = P.token_logprobs(x, tok, 1)
    want = 5 - math.log(V - 1 + math.exp(5))
    for i, r in enumerate(at):
        assert abs(lp[r].item() - want) <= 1e-6 and idx[r].item() == 1000 + i
    assert lp.count_nonzero().item() == 3 and (idx != -1).sum().item() == 3


def check32(got, x, tokens, k, tau=1.0, rows=None):
    """check(), of values that may leave fp32's range (their rounding is -inf) and of rows with several
    largest entries.  Those stay in a wave's sums where they make up half of them or more: their terms are
    rounded as the others' (ref64_samples.logprobs: 6 * 3 + 4 + 129 + 6 + 15 roundings), and so is
    what they weigh in the entropy, whose exponents are then the rounding of a reference below 2^20."""
    lp, ent, idx, val = [None if t is None else t.double().cpu() for t in got]
    f32 = lambda v: torch.tensor(v, dtype=torch.float64).float().item()  # noqa: E731
    x = x.cpu()
    for r, t in enumerate(tokens):
        if t < 0:
            continue
        w_lp, w_ent, order, top, e_lp, e_ent = R.logprobs(x[r if rows is None else rows[r]], tau, t, k)
        d = (x[r if rows is None else rows[r]].double() - x[r if rows is None else rows[r]].double().max()) / tau
        n = (d == 0).sum().item()
        tops = n * 172 * 2.0 ** -24 / torch.exp(d).sum().item() if n > 1 else 0.0
        e_lp, e_ent = e_lp + tops, e_ent + tops * (2 + w_ent)
        assert lp[r] == f32(w_lp) or abs(lp[r] - w_lp) <= e_lp + 2.0 ** -24 * abs(w_lp), (r, lp[r], w_lp, e_lp)
        assert abs(ent[r] - w_ent) <= e_ent, (r, ent[r], w_ent, e_ent)
        if k:
            assert idx[r].int().tolist() == order, (r, idx[r].tolist(), order)
            for a, b in zip(val[r].tolist(), top):
                assert a == f32(b) or abs(a - b) <= e_lp + 2.0 ** -24 * abs(b), (r, a, b, e_lp)


def low_rows(V, dtype, what, seed):
    """Rows whose logits, or most of them, lie far below 0: (row, temperature) of every kind of one test."""
    g = torch.Generator("cuda").manual_seed(seed)
    lowest = torch.finfo(dtype).min
    ordinary = lambda: torch.randn(V, generator=g, device="cuda") * 2  # noqa: E731
    got = []
    if what == "masks":  # finite masks, a few tokens allowed
        for mask in (-1e4, -65504.0, -1e5, -1e6, -1e7, -1e8, -7e8, -1e9, lowest):
            for allowed in (1, 3, 50):
                x = torch.full((V,), mask, device="cuda")
                at = torch.randperm(V, generator=g, device="cuda")[:allowed]
                x[at] = torch.randn(len(at), generator=g, device="cuda") * 2
                got.append((x, 1.0))
            x = ordinary()
            x[: V // 2] = mask                  # whole slices
            got.append((x, 1.0))
            x = ordinary()
            x[V - V // 8 - 1:] = mask           # a padded end of the vocabulary
            got.append((x, 0.7))
    elif what == "uniform":  # nothing allowed
        for mask in (-65504.0, -1e6, -1e7, -1e8, -7e8, -1e9, lowest):
            got.append((torch.full((V,), mask, device="cuda"), 1.0))
        got += [(torch.full((V,), -65504.0, device="cuda"), t) for t in (0.07, 0.02, 1e-4)]
    elif what == "low":  # all logits far below 0, near each other and not
        for base in (-1e5, -1e6, -1e7, -1e8, -7e8, -1e9):
            for spread in (2.0 ** -21, 2.0 ** -16, 2.0 ** -8, 1.0):
                got.append((base * (1 + spread * torch.rand(V, generator=g, device="cuda")), 1.0))
    else:  # low temperatures on negative logits
        for tau in (0.05, 1e-3, 2e-5, 1e-5, 1e-6, 1e-7, 1e-30):
            for top in (-0.01, -3.0, -20.0, -35.0):
                got.append((top - torch.rand(V, generator=g, device="cuda") * 5, tau))
            x = -3 - torch.rand(V, generator=g, device="cuda")
            x[: min(V, 40)] = -3.0
            got.append((x, tau))
    return [(x.to(dtype), tau) for x, tau in got]


# few rows: one slice, several; many of them: a wave per row
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("what", ["masks", "uniform", "low", "cold"])
@pytest.mark.parametrize("V,N,k", [(300, 1, 8), (1000, 700, 8), (1000, 1, 0), (2100, 4200, 16), (20000, 1, 8), (66003, 1, 5)])
def test_low_references(P, dtype, what, V, N, k):
    rows = low_rows(V, dtype, what, V)
    r = random.Random(V)
    for tau in sorted({t for _, t in rows}):
        x = torch.stack([y for y, t in rows if t == tau])
        m = x.shape[0]
        tok = [[y.argmax().item(), r.randrange(V), y.argmin().item()][i % 3] for i, y in enumerate(x)]
        n = -(-N // m)
        st = i32([0])
        got = P.token_logprobs(x.repeat(n, 1), i32(tok * n), k, temperature=tau, dev_status=st)
        assert st.item() == 0
        check32([None if t is None else t[-m:] for t in got], x, tok, k, tau)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [500, 40000])
def test_low_references_along_paths(P, dtype, V):
    for what in ("masks", "uniform", "cold"):
        for tau in (1.0, 1e-5):
            rows = [y for y, t in low_rows(V, dtype, what, V + 1) if t == tau]
            if not rows:
                continue
            T = 6
            x = torch.stack((rows * (T + 1))[: 2 * (T + 1)])
            nodes, n = [[0, 2, 5, -1, -1, -1], [1, -1, -1, -1, -1, -1]], [3, 1]
            tok = [j * 7 if j <= n[b] else -1 for b in range(2) for j in range(T + 1)]
            at = [b * (T + 1) + (nodes[b][j - 1] + 1 if 0 < j <= n[b] else 0) for b in range(2) for j in range(T + 1)]
            got = P.token_logprobs(x.view(2, T + 1, V), i32(tok), 4, nodes=i32(nodes), temperature=tau)
            check32(got, x, tok, 4, tau, rows=at)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,N", [(1000, 1), (32768, 130)])
def test_rows_in_order_far_below_zero(P, dtype, V, N):
    # the reference moves with every group of chunks where the type's steps are many doublings
    rows = []
    for base, span in ((-1000.0, 200.0), (-5056.0, 700.0), (-20000.0, 3000.0), (-60000.0, 9000.0), (-300.0, 20.0)):
        up = (base + torch.linspace(0, span, V, device="cuda")).to(dtype)
        rows += [up, up.flip(0)]
        x = torch.full((V,), -math.inf, dtype=dtype, device="cuda")  # one entry, and two at the end, a step of bf16 larger
        x[0] = base
        x[V - 2:] = torch.nextafter(torch.tensor(base, dtype=torch.bfloat16), torch.tensor(0.0, dtype=torch.bfloat16)).item()
        rows.append(x)
    x = torch.stack(rows * N)
    tok = [0, V - 1, V - 2] * (len(rows) // 3)
    for tau in (1.0, 0.6, 7.0):
        got = P.token_logprobs(x, i32(tok * N), 8, temperature=tau)
        check32([t[:len(rows)] for t in got], x[:len(rows)], tok, 8, tau)
        for t in got:
            assert torch.equal(t.view(N, -1), t.view(N, -1)[:1].expand(N, -1))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,N", [(40, 1), (1000, 1), (20000, 1), (128256, 1), (700, 260)])
def test_every_rank_of_rows_of_no_numbers(P, dtype, V, N):
    # NaN with the sign set, a few numbers or -inf among them: indices of the row, each once, the numbers first
    # (as a pattern: a conversion may lose a NaN's sign)
    x = (torch.full((5, V), -0x40, dtype=torch.int16, device="cuda") if dtype == torch.bfloat16 else
         torch.full((5, V), -0x400000, dtype=torch.int32, device="cuda")).view(dtype)
    x[1, 7], x[1, V - 1] = 2.0, 3.0
    x[2, ::2] = -math.inf
    x[3, : V // 2] = -math.inf
    x[4, V // 2:] = torch.linspace(-1, 1, V - V // 2, device="cuda")
    _, _, idx, _ = P.token_logprobs(x.repeat(N, 1), None, 5)
    assert torch.equal(idx.view(N, 5, 5), idx[:5].expand(N, 5, 5))
    assert ((idx >= 0) & (idx < V)).all() and all(len(set(row)) == 5 for row in idx[:5].tolist())
    assert idx[1, :2].tolist() == [V - 1, 7] and (idx[4] >= V // 2).all()
