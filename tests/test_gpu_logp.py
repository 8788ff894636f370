"""GPU parity of the token log-probabilities and of the logits' gradient against the fp64 oracle.

Tolerances (u = 2^-24, half a step of fp32).  l = log S, S a sum of V powers of two, each within 4 u from the function
(2^-22) and u times its exponent's size from the argument's rounding; the part of a term with exponent -e is 2^-e / S, so that
those errors add up to less than u (16 + 2 |l|).  A thread adds at most 512 terms one after the other (a row of 8 KB by one
warp, or one of 256 KB by 512 threads in two sums) and the joins 16 more: u 528.  logp = (x_y - m) / temperature - l adds
three roundings of its parts.  So |error| <= u (600 + 8 |l| + 8 |x_y - m| / temperature).
The gradient's element g p: the exponent's argument, up to E = |m + l| log2(e) before K is taken off, comes from c x with c = log2(e)
/ temperature rounded and m rounded once more: u (32 + 4 E) of itself, and l's own error above; then
half a step of the logits' type, and of its smallest number."""
import numpy as np
import pytest
import torch

from oracle import policy as P
from paper_2602_24082_b200 import workloads as W

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -126), "fp16": (torch.float16, 2.0 ** -11, 2.0 ** -25),
         "fp32": (torch.float32, U, 2.0 ** -126)}

STRUCTURES = {
    "pair": [[(64, (32, 48))]],
    "ragged": [[(57, (5, 28, 31))], [(1, (1, 30))]],
    "ones": [[(1, (1,) * 37)], [(2, (1,))]],
    "single": [[(9, (1,)), (1, (17,))]],
    "one_token": [[(1, (1,))]],
}


def _plan(rows, **kw):
    from paper_2602_24082_b200 import binding as B
    return B.plan_for(W.Workload("logp", rows, 2, 1, 64, seed=0), **kw)


def _inputs(rows, V, dtype, seed, stride=None, offset=0, ids_dtype=torch.int64):
    T = sum(p + sum(rs) for row in rows for p, rs in row)
    g = torch.Generator().manual_seed(seed)
    x = 3 * torch.randn(T, V, generator=g)
    ids = torch.randint(0, V, (T,), generator=g)
    for r, t in P.predictions(rows):
        if torch.rand((), generator=g) < 0.7:
            x[r, ids[t]] += 12 * torch.rand((), generator=g)
    stride = stride or V
    buf = torch.full((T * stride + offset,), float("nan"), dtype=dtype, device="cuda")
    view = buf[offset:].as_strided((T, V), (stride, 1))
    view.copy_(x.to(dtype))
    return view, ids.to(ids_dtype).cuda(), buf


def _f64(t):
    return t.double().cpu().numpy()


def _check_fwd(rows, logits, ids, temperature, logp, stats):
    x, y = _f64(logits), ids.cpu().numpy()
    temp = float(np.float32(temperature))
    want, st = P.token_logp(rows, x, y, temp)
    logp, stats = _f64(logp), _f64(stats)
    assert np.array_equal(np.isnan(logp), np.isnan(want))
    l = np.zeros(len(want))
    for r, t in P.predictions(rows):
        l[t] = st[r, 1]
    tol = U * (600 + 8 * np.abs(l) + 8 * np.abs(want + l))
    fine = np.isfinite(want)
    assert np.array_equal(logp[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
    assert (np.abs(logp - want)[fine] <= tol[fine]).all(), np.abs(logp - want)[fine].max()
    used = st.any(1)
    assert not stats[~used].any()
    assert (np.abs(stats - st)[:, 0] <= U * np.abs(st[:, 0])).all()
    assert (np.abs(stats - st)[:, 1] <= U * (600 + 8 * np.abs(st[:, 1]))).all()


def _check_bwd(rows, logits, ids, grad, temperature, d, kind):
    _, half, tiny = TYPES[kind]
    temp = float(np.float32(temperature))
    x = _f64(logits)
    want, size = P.token_logp_bwd(rows, x, ids.cpu().numpy(), _f64(grad), temp)
    top = np.where(np.isfinite(x).any(1), np.where(np.isfinite(x), x, -np.inf).max(1), 0)
    E = np.abs(top / temp) * 1.4427
    E = np.where(E < 2.0 ** 19, E, 0) + np.log2(x.shape[1] + 1)      # (beyond, exp(x - m - l) itself is taken)
    # the power 2^(c x - K) is 0 below 2^-126 (flushed); the row's factor, at most the sum of |g| / temperature times
    # 2^(1/2) for the fraction taken off with K, multiplies it: that much is lost, whatever the type
    weight = np.zeros(len(x))
    np.add.at(weight, [r for r, _ in P.predictions(rows)], np.abs(_f64(grad))[[t for _, t in P.predictions(rows)]])
    flushed = 2.0 ** -126 * 1.4143 * weight / temp
    tol = half * np.abs(want) * (1 + 2 * half) + U * (700 + 8 * E)[:, None] * size + tiny + flushed[:, None]
    err = np.abs(_f64(d) - want)
    assert (err <= tol).all(), (err / tol).max()


VOCABS = [1, 2, 7, 8, 31, 257, 1000, 2048, 4099, 8200, 16391, 33000]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("structure", list(STRUCTURES))
def test_parity(structure, V, kind):
    from paper_2602_24082_b200 import binding as B
    rows, seed = STRUCTURES[structure], V + len(structure)
    layout = [dict(), dict(stride=V + 5), dict(offset=1), dict(stride=V + 8 - V % 8, ids_dtype=torch.int32)][seed % 4]
    temperature = [1.0, 0.7][seed % 2]
    logits, ids, buf = _inputs(rows, V, TYPES[kind][0], seed, **layout)
    plan = _plan(rows, desc_on_device=seed % 3 == 0)
    logp, stats = B.pp_token_logp(plan, logits, ids, temperature)
    g = torch.randn(len(ids), generator=torch.Generator().manual_seed(seed)).cuda()
    d = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g, temperature)
    # ... into rows that lie otherwise than the logits', with room behind them
    other = torch.full((len(ids), V + 3), 5.0, dtype=logits.dtype, device="cuda")
    B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g, temperature, d_logits=other[:, :V])
    torch.cuda.synchronize()
    assert plan.status() == (0, 0)
    assert d.stride(0) == logits.stride(0) or len(ids) == 1
    _check_fwd(rows, logits, ids, temperature, logp, stats)
    _check_bwd(rows, logits, ids, g, temperature, d, kind)
    _check_bwd(rows, logits, ids, g, temperature, other[:, :V], kind)
    assert (other[:, V:] == 5).all()
    # in place, and what lies between the rows stays
    before = buf.clone()
    B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g, temperature, d_logits=logits)
    assert torch.equal(logits, d)
    logits.copy_(before[layout.get("offset", 0):].as_strided(logits.shape, logits.stride()))
    assert torch.equal(buf.view(torch.uint8), before.view(torch.uint8))


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("V", [50257, 128256])
@pytest.mark.parametrize("tokens", ["few", "more", "many"])
def test_parity_of_large_vocabularies(tokens, V, kind):
    """Rows that 8, 4, 2 and 1 blocks share, and those of 128 threads."""
    from paper_2602_24082_b200 import binding as B
    rows = {"few": [[(3, (2, 1))]], "more": [[(90, (20, 12))], [(60, (9,))]], "many": [[(700, (7, 5, 2))]]}[tokens]
    logits, ids, _ = _inputs(rows, V, TYPES[kind][0], 3)
    plan = _plan(rows)
    g = torch.randn(len(ids), generator=torch.Generator().manual_seed(5)).cuda()
    logp, stats = B.pp_token_logp(plan, logits, ids)
    d = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g)
    assert plan.status() == (0, 0)
    used = sorted({r for r, _ in P.predictions(rows)})
    assert not torch.cat([d[i:i + 1] for i in range(len(ids)) if i not in set(used)]).any()
    _check_fwd(rows, logits, ids, 1.0, logp, stats)
    _check_bwd(rows, logits, ids, g, 1.0, d, kind)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [600, 9001, 20000])
def test_parity_of_mostly_prompts(V, kind):
    """Few rows that predict something; the others are not read."""
    from paper_2602_24082_b200 import binding as B
    rows = [[(1200, (40, 30, 9))], [(90, (3,)), (1, (1, 2))]]
    logits, ids, _ = _inputs(rows, V, TYPES[kind][0], 7)
    ids[[1200, 1370]] = -1
    used = sorted({r for r, t in P.predictions(rows) if ids[t] >= 0})
    logits[[i for i in range(len(ids)) if i not in set(used)]] = float("nan")      # not read
    g = torch.randn(len(ids), generator=torch.Generator().manual_seed(5)).cuda()
    for on_device in (False, True):
        plan = _plan(rows, desc_on_device=on_device)
        logp, stats = B.pp_token_logp(plan, logits, ids)
        d = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g)
        assert plan.status() == (0, 0)
        safe = torch.nan_to_num(logits)
        _check_fwd(rows, safe, ids, 1.0, logp, stats)
        _check_bwd(rows, safe, ids, g, 1.0, d, kind)


@pytest.mark.parametrize("V,rows", [(257, [[(2, (30, 31)), (40, (1, 2, 3))]] * 48), (3000, [[(2, (30, 31)), (40, (1, 2, 3))]] * 48),
                                    (31, [[(2, (3, 1)), (1, (1,))]] * 1100)], ids=["257", "3000", "segments"])
def test_parity_of_many_short_rows(V, rows):
    from paper_2602_24082_b200 import binding as B
    logits, ids, _ = _inputs(rows, V, torch.bfloat16, 9)
    assert len(ids) > 32 * 148
    plan = _plan(rows)
    g = torch.randn(len(ids), generator=torch.Generator().manual_seed(5)).cuda()
    logp, stats = B.pp_token_logp(plan, logits, ids)
    d = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g)
    _check_fwd(rows, logits, ids, 1.0, logp, stats)
    _check_bwd(rows, logits, ids, g, 1.0, d, "bf16")


@pytest.mark.parametrize("T,V", [(20000, 17000), (40000, 5001), (9600, 66000), (12345, 66001)])
def test_the_way_rows_are_dealt_out_does_not_change_them(T, V):
    """A plan from host arrays knows how many tokens the responses hold, one from device arrays does not: their
    blocks look over other numbers of rows."""
    from paper_2602_24082_b200 import binding as B
    rows = [[(T - 310, (200, 7))], [(2, (1, 100))]]
    g = torch.Generator(device="cuda").manual_seed(0)
    logits = torch.randn(T, V, generator=g, device="cuda", dtype=torch.bfloat16)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    a, b = (B.pp_token_logp(_plan(rows, desc_on_device=d), logits, ids) for d in (False, True))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and a[0].count_nonzero() > 300
    r, t = (torch.tensor(x, device="cuda") for x in zip(*P.predictions(rows)))
    want = torch.log_softmax(logits[r].double(), -1)[torch.arange(len(t), device="cuda"), ids[t]]
    assert float((a[0][t].double() - want).abs().max()) < U * (600 + 8 * 12 + 8 * 30)


@pytest.mark.parametrize("V,kind", [(100, "fp32"), (4099, "bf16"), (20000, "fp16"), (60000, "fp32"), (140000, "bf16")])
def test_masked_and_extreme_logits(V, kind):
    from paper_2602_24082_b200 import binding as B
    rows = [[(5, (6, 4, 3))], [(2, (9,))]]
    dtype, lowest = TYPES[kind][0], torch.finfo(TYPES[kind][0]).min
    logits, ids, _ = _inputs(rows, V, dtype, 1)
    x = logits
    x[:4] = float("nan")                       # rows that predict nothing are not read
    x[10] = float("inf")                       # (the end of the first response)
    x[4, V // 3:] = -float("inf")              # ids that cannot be sampled ...
    ids[5] = V - 1                             # ... of which one was
    x[5, :] = -float("inf")
    x[5, V // 2] = -3.0                        # a single one left
    ids[6] = V // 2
    x[6] = lowest                              # nothing left: all alike
    x[7] = lowest
    x[7, 1] = 2.5
    x[8] = -float("inf")                       # nothing at all
    x[9, V - 1] = float("inf")
    x[11, 0] = float("nan")
    x[12] = lowest / 2
    x[12, V - 2] = lowest / 4
    ids[13] = V - 2
    ids[16] = -1
    ids[17] = V
    plan = _plan(rows)
    logp, stats = B.pp_token_logp(plan, logits, ids)
    want, st = P.token_logp(rows, _f64(x), ids.cpu().numpy())
    got = _f64(logp)
    assert got[5] == -np.inf and abs(got[7] + np.log(V)) <= U * 700
    # (certain tokens: 0 but for the bound above with l = 0 and x_y = m; fp16's lowest, -65504, is not far enough for exact terms)
    assert abs(got[6]) <= U * 600 and abs(got[13]) <= U * 600
    assert np.isnan(got[9:11]).all() and np.isnan(got[12]) and got[16] == 0 and np.isnan(got[17])
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    fine = np.isfinite(want)
    assert (np.abs(got[fine] - want[fine]) <= U * (600 + 8 * np.log(V) + 8 * np.abs(want[fine]))).all()
    # gradients of the rows that are numbers
    g = torch.randn(len(ids), generator=torch.Generator().manual_seed(5)).cuda()
    g[torch.from_numpy(nan).cuda()] = 0
    d = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g)
    assert plan.status() == (0, 0)
    safe = torch.where(torch.isnan(x) | (x == float("inf")), torch.zeros_like(x), x)
    safe[8] = 0
    _check_bwd(rows, safe, ids, g, 1.0, d, kind)


@pytest.mark.parametrize("V", [300, 5000, 20000, 140000])
def test_rows_that_rise_fall_and_jump(V):
    """A thread's reference comes from its first elements: rows whose later ones are larger by less and by more than
    the 2^64 that it may stay for, at the end, in the middle, everywhere."""
    from paper_2602_24082_b200 import binding as B
    rows = [[(1, (12, 9))]]
    logits, ids, _ = _inputs(rows, V, torch.float32, 3)
    x, n = logits, torch.linspace(0, 1, V, device="cuda")
    x[0] = 800 * n - 400
    x[1] = 400 - 800 * n
    x[2] = -30.0 + 1e-3 * x[2]
    x[2, V - 1] = 12.0                  # 2^61 times as large
    x[3] = -30.0 + 1e-3 * x[3]
    x[3, V // 2] = 17.0                 # 2^68
    x[4] = -3000.0 * (n < 0.5) + 0.01 * x[4]
    x[5] = -60.0 * (1 - n)
    x[6] = 1000 * torch.sin(40 * n)
    x[7] = 0.0
    x[8] = torch.where(torch.arange(V, device="cuda") % 2 == 0, 44.0, -44.0)
    x[9, : V - 1] = -float("inf")
    x[10] = -float("inf")
    x[10, V // 3] = 300000.0
    x[11, 0] = 3000.0
    for t, y in ((2, V - 1), (3, V - 1), (4, V // 2), (5, V - 1), (10, V - 1), (11, V // 3), (14, 0)):
        ids[t] = y
    plan = _plan(rows)
    logp, stats = B.pp_token_logp(plan, logits, ids)
    g = torch.randn(len(ids), generator=torch.Generator().manual_seed(5)).cuda()
    d = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g)
    _check_fwd(rows, logits, ids, 1.0, logp, stats)
    _check_bwd(rows, logits, ids, g, 1.0, d, "fp32")


@pytest.mark.parametrize("V", [300, 20000, 60000])
@pytest.mark.parametrize("offset", [-4096.0, 30000.0])
def test_an_offset_of_all_logits_costs_nothing(V, offset):
    """Logits on a grid of 2^-8, which stay what they are with the offset: everything is relative to the row's maximum, so
    the bounds are those of logits around zero, without the term for the exponent's size."""
    from paper_2602_24082_b200 import binding as B
    rows = [[(2, (12, 9, 1))]]
    logits, ids, _ = _inputs(rows, V, torch.float32, 3)
    logits.copy_((logits * 256).round() / 256)
    plan = _plan(rows)
    g = torch.randn(len(ids), generator=torch.Generator().manual_seed(5)).cuda()
    moved = logits + offset
    assert torch.equal(moved - offset, logits)
    logp, stats = B.pp_token_logp(plan, moved, ids)
    d = B.pp_token_logp_bwd(plan, moved, ids, logp, stats, g)
    stats[:, 0] -= offset * (stats[:, 0] != 0)
    _check_fwd(rows, logits, ids, 1.0, logp, stats)
    _check_bwd(rows, logits, ids, g, 1.0, d, "fp32")


@pytest.mark.parametrize("V", [50, 5000, 70000])
def test_the_same_id_of_several_responses_and_gradients_that_cancel(V):
    from paper_2602_24082_b200 import binding as B
    rows = [[(3, (2, 1, 4, 1, 1))], [(4, (1,) * 70)]]
    logits, ids, _ = _inputs(rows, V, torch.float32, 2)
    seqs = P.sequences(rows)
    first = [y[0] for y in seqs[0][1]]
    ids[first] = torch.tensor([7, 7, 9, -1, 7]).cuda()
    ids[[y[0] for y in seqs[1][1]]] = torch.arange(70).cuda() % 3
    g = torch.randn(len(ids), generator=torch.Generator().manual_seed(1)).cuda()
    g[first] = torch.tensor([1.0, -3.0, 2.0, 9.0, 0.0]).cuda()      # those that count add up to zero
    plan = _plan(rows)
    logp, stats = B.pp_token_logp(plan, logits, ids)
    d = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g)
    _check_fwd(rows, logits, ids, 1.0, logp, stats)
    _check_bwd(rows, logits, ids, g, 1.0, d, "fp32")


def test_rows_without_a_gradient_are_not_read():
    from paper_2602_24082_b200 import binding as B
    rows = [[(3, (4, 2))]]
    logits, ids, _ = _inputs(rows, 3000, torch.bfloat16, 4)
    plan = _plan(rows)
    logp, stats = B.pp_token_logp(plan, logits, ids)
    g = torch.zeros(len(ids), device="cuda")
    g[4] = 1.0
    logits[[0, 1, 2, 4, 5, 6, 7, 8]] = float("nan")
    d = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g)
    assert not d[[0, 1, 2, 4, 5, 6, 7, 8]].any() and d[3].float().abs().sum() > 0.1


def test_gradient_against_differences():
    """The log-probabilities of the kernel itself, moved by h in a direction: their sum's slope is the gradient's
    product with it.  Differences of fp32 values of size 10: 2 u 600 / h, and h^2 for the curvature."""
    from paper_2602_24082_b200 import binding as B
    rows = [[(3, (4, 2, 1))], [(5, (3,))]]
    logits, ids, _ = _inputs(rows, 700, torch.float32, 6)
    plan = _plan(rows)
    g = torch.randn(len(ids), generator=torch.Generator().manual_seed(2)).cuda()
    logp, stats = B.pp_token_logp(plan, logits, ids, 0.7)
    d = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g, 0.7).double()
    h = 2.0 ** -7
    for seed in range(4):
        v = torch.randn(logits.shape, generator=torch.Generator().manual_seed(seed)).cuda()
        up, down = (B.pp_token_logp(plan, logits + s * h * v, ids, 0.7)[0].double() for s in (1, -1))
        slope = ((up - down) * g.double()).sum() / (2 * h)
        assert abs(float(slope - (d * v.double()).sum())) < float(g.abs().sum()) * (U * 700 / h + 8 * h * h)


def test_offsets_beyond_32_bits():
    """34000 rows of 131072 columns: elements beyond 2^32."""
    from paper_2602_24082_b200 import binding as B
    rows, V = [[(100, (4, 6))], [(33000, (400, 490))]], 131072
    T = 34000
    logits = torch.zeros(T, V, dtype=torch.bfloat16, device="cuda")
    at = torch.arange(33105, T, 7, device="cuda")
    at = torch.cat([torch.tensor([99, 101, 33109], device="cuda"), at])
    logits[at] = torch.randn(len(at), V, generator=torch.Generator(device="cuda").manual_seed(0), device="cuda").bfloat16()
    ids = (torch.arange(T, device="cuda") * 977) % V
    plan = _plan(rows)
    logp, stats = B.pp_token_logp(plan, logits, ids)
    g = torch.ones(T, device="cuda")
    d = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g, d_logits=logits)
    assert d.data_ptr() == logits.data_ptr() and plan.status() == (0, 0)
    for r, t in P.predictions(rows)[-60:]:
        x = torch.zeros(V, dtype=torch.float64, device="cuda")
        k = (at == r).nonzero()
        if len(k):
            x = torch.randn(len(at), V, generator=torch.Generator(device="cuda").manual_seed(0), device="cuda").bfloat16()[int(k[0])].double()
        lp = torch.log_softmax(x, 0)
        y = int(ids[t])
        assert abs(float(logp[t] - lp[y])) < 2e-4
        want = -lp.exp()
        want[y] += 1
        assert float((d[r].double() - want).abs().max()) < 2.0 ** -8


@pytest.mark.parametrize("V", [300, 20000, 128256])
def test_streams_graphs_and_repeats(V):
    """The same bits every time: again, on another stream, and replayed from a graph on new inputs."""
    from paper_2602_24082_b200 import binding as B
    rows = [[(40, (9, 20, 1))], [(3, (30,))]]
    logits, ids, _ = _inputs(rows, V, torch.bfloat16, 8)
    plan = _plan(rows)
    g = torch.randn(len(ids), device="cuda")

    def step():
        logp, stats = B.pp_token_logp(plan, logits, ids)
        return logp, stats, B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g)

    want = step()
    assert all(torch.equal(a, b) for a, b in zip(step(), want))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        there = step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            held = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(there, want))
    logits.copy_(torch.roll(logits, 1, 1))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, step()))
    assert not torch.equal(held[0], want[0])


def test_given_outputs():
    from paper_2602_24082_b200 import binding as B
    rows = [[(3, (4, 2))]]
    logits, ids, _ = _inputs(rows, 1000, torch.float16, 1)
    plan = _plan(rows)
    logp, stats = B.pp_token_logp(plan, logits, ids)
    a, b = torch.full((9,), 5.0, device="cuda"), torch.full((9, 2), 5.0, device="cuda")
    for kw in (dict(token_logp=a), dict(row_stats=b), dict(token_logp=a, row_stats=b)):
        a.fill_(5), b.fill_(5)
        got = B.pp_token_logp(plan, logits, ids, **kw)
        assert torch.equal(got[0], logp) and torch.equal(got[1], stats)
        assert got[0] is kw.get("token_logp", got[0]) and got[1] is kw.get("row_stats", got[1])
    for bad in (dict(token_logp=a[:-1]), dict(token_logp=a.half()), dict(row_stats=b.T), dict(row_stats=b.cpu())):
        with pytest.raises(ValueError):
            B.pp_token_logp(plan, logits, ids, **bad)
    # what the call returns lies side by side in one allocation: writing to one leaves the others as they are
    logp.fill_(3)
    assert torch.equal(stats, b)


def test_refusals():
    from paper_2602_24082_b200 import binding as B
    rows = [[(3, (4, 2))]]
    logits, ids, _ = _inputs(rows, 100, torch.bfloat16, 1)
    plan = _plan(rows)
    logp, stats = B.pp_token_logp(plan, logits, ids)
    for bad in (logits[:-1], logits.double(), logits.T, logits.cpu(), logits[:, ::2], logits[0], logits[:, :0]):
        with pytest.raises(ValueError):
            B.pp_token_logp(plan, bad, ids)
    for bad in (ids[:-1], ids.float(), ids.cpu(), ids[::2]):
        with pytest.raises(ValueError):
            B.pp_token_logp(plan, logits, bad)
    for t in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(B.PPError):
            B.pp_token_logp(plan, logits, ids, t)
    g = torch.ones(9, device="cuda")
    for bad in (dict(d_logits=logits.float()), dict(d_logits=logits[:, :50]), dict(d_logits=logits[:5])):
        with pytest.raises(ValueError):
            B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g, **bad)
    for args in ((logp[:-1], stats, g), (logp, stats.T, g), (logp, stats, g.double()), (logp, stats, g.cpu())):
        with pytest.raises(ValueError):
            B.pp_token_logp_bwd(plan, logits, ids, *args)


# A warp, 128 threads, 256 threads and several blocks take a row of the gradient.
BACKWARD_SHAPES = [(100, [[(5, (700, 600))]]), (5000, [[(5, (700, 600))]]), (300, [[(2, (12, 9, 1))]]), (20000, [[(2, (12, 9, 1))]]),
                   (140000, [[(2, (12, 9, 1))]])]
BACKWARD_IDS = ["warp", "four_warps", "few", "two_blocks", "eight_blocks"]


@pytest.mark.parametrize("V,rows", BACKWARD_SHAPES, ids=BACKWARD_IDS)
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("temperature", [0.7, 1.0, 1.3])
def test_rows_far_from_zero_at_any_temperature(V, rows, kind, temperature):
    """Rows at the ends of the type's range, whose maximum over the temperature may pass fp32's: log-probabilities and
    gradients are those relative to the maximum (the bounds without the term for the exponent's size), in place too."""
    from paper_2602_24082_b200 import binding as B
    dtype, lowest = TYPES[kind][0], torch.finfo(TYPES[kind][0]).min
    logits, ids, _ = _inputs(rows, V, dtype, 1)
    x, n = logits, torch.arange(V, device="cuda")
    first = rows[0][0][0]                      # the first response's rows
    near = torch.tensor(lowest, device="cuda").to(dtype) * 0.75
    x[first] = lowest
    x[first + 1] = -lowest
    x[first + 2] = torch.where(n % 3 == 1, near, x[first])          # all of them beyond 0.7 of the range
    x[first + 3] = torch.where(n % 7 == 2, -near, x[first])
    x[first + 4] = torch.where(n == V - 1, 2.5, lowest)
    x[first + 5] = torch.where(n < V // 2, -torch.inf, near)
    ids[first + 1: first + 7] = torch.tensor([0, 0, 1, 2, 0, V - 1]).cuda()
    plan = _plan(rows)
    logp, stats = B.pp_token_logp(plan, logits, ids, temperature)
    # the same rows relative to their maximum, in 64 bits
    safe = logits.double() - logits.double().amax(1, keepdim=True)
    temp = float(np.float32(temperature))
    want, st = P.token_logp(rows, _f64(safe), ids.cpu().numpy(), temp)
    got = _f64(logp)
    l = np.zeros(len(want))
    for r, t in P.predictions(rows):
        l[t] = st[r, 1]
    tol = U * (600 + 8 * np.abs(l) + 8 * np.abs(want + l))
    # (beyond fp32's largest number a log-probability is -inf)
    assert (np.abs(got - want) <= tol)[np.abs(want) < 3e38].all()
    assert (got[np.abs(want) > 3.5e38] == -np.inf).all()
    assert np.isfinite(_f64(stats)[:, 1]).all()
    g = torch.randn(len(ids), generator=torch.Generator().manual_seed(5)).cuda()
    d = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g, temperature)
    _check_bwd(rows, safe, ids, g, temperature, d, kind)
    other = torch.full((len(ids), V + 3), 5.0, dtype=dtype, device="cuda")
    B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g, temperature, d_logits=other[:, :V])
    assert torch.equal(other[:, :V], d)
    assert torch.equal(B.pp_token_logp_bwd(plan, logits, ids, logp, stats, g, temperature, d_logits=logits), d)


@pytest.mark.parametrize("V,rows", BACKWARD_SHAPES, ids=BACKWARD_IDS)
@pytest.mark.parametrize("kind,offset,grid", [("fp32", 200.0, 2.0 ** -12), ("fp32", -4096.0, 2.0 ** -8), ("fp32", 30000.0, 2.0 ** -8), ("fp32", 3e6, 0.25),
                                              ("fp16", 800.0, 0.5), ("fp16", -30000.0, 16.0), ("bf16", -800.0, 4.0),
                                              ("bf16", 196608.0, 1024.0), ("bf16", 3145728.0, 16384.0)])
@pytest.mark.parametrize("temperature", [0.7, 1.3, 0.01, 1e-4])
def test_an_offset_costs_nothing_at_a_temperature(V, rows, kind, offset, grid, temperature):
    """Logits on the type's grid around an offset.  row_stats hold the maximum over the temperature, rounded to fp32: for
    16-bit logits the maximum itself follows from it, fp32 rows far from zero are read again, so the bounds are those of logits
    whose maximum is zero.  Of other fp32 rows the gradient has that rounding, u |m| / temperature, for a factor."""
    from paper_2602_24082_b200 import binding as B
    logits, ids, _ = _inputs(rows, V, torch.float32, 3)
    base = (logits * max(1.0, temperature) * (1 if grid < 1 else grid / 2) / grid).round() * grid
    moved = (base + offset).to(TYPES[kind][0])
    assert torch.equal(moved.double() - offset, base.double())
    safe = base.double() - base.double().amax(1, keepdim=True)
    plan = _plan(rows)
    logp, stats = B.pp_token_logp(plan, moved, ids, temperature)
    g = 0.25 * torch.randn(len(ids), generator=torch.Generator().manual_seed(5)).cuda()      # (over 1e-4: within fp16's range)
    d = B.pp_token_logp_bwd(plan, moved, ids, logp, stats, g, temperature)
    temp = float(np.float32(temperature))
    want, st = P.token_logp(rows, _f64(safe), ids.cpu().numpy(), temp)
    l = np.zeros(len(want))
    for r, t in P.predictions(rows):
        l[t] = st[r, 1]
    assert (np.abs(_f64(logp) - want) <= U * (600 + 8 * np.abs(l) + 8 * np.abs(want + l))).all()
    top = float(base.amax()) + abs(offset)
    if kind == "fp32" and top / temp * 1.4427 < 512:
        # (a factor 1 + e of the probabilities, e <= u |m| / temperature)
        want, size = P.token_logp_bwd(rows, _f64(safe), ids.cpu().numpy(), _f64(g), temp)
        assert (np.abs(_f64(d) - want) <= U * (700 + 8 * np.log2(V + 1) + 2 * top / temp) * size + 2.0 ** -120).all()
    else:
        _check_bwd(rows, safe, ids, g, temperature, d, kind)
    assert torch.equal(B.pp_token_logp_bwd(plan, moved, ids, logp, stats, g, temperature, d_logits=moved), d)


@pytest.mark.parametrize("V", [600, 5000, 50257, 128256])
@pytest.mark.parametrize("temperature", [1.0, 0.7])
@pytest.mark.parametrize("kind", list(TYPES))
def test_certain_tokens(V, temperature, kind):
    """One column far above the others, in every part of the row.  log p = -log1p(sum of the others), to within u times
      4    the power of that column (2^-22),
      2.8  its exponent, at most 8 above the reference: half a step of 4 .. 8, 2^-22, times log 2,
      1.5  log S (one step of up to log 2) and what is left of the maximum behind the reference (half a step of 1),
    and the others' share, of which sums may lose any part.  (64 above the reference were 22 u.)"""
    from paper_2602_24082_b200 import binding as B
    n = 60
    rows = [[(1, (n,))]]
    g = torch.Generator().manual_seed(V)
    x = torch.randn(n + 1, V, generator=g).clamp(-3, 3)
    ids = torch.randint(0, V, (n + 1,), generator=g)
    peak = temperature * torch.linspace(20, 70, n, dtype=torch.float64)
    x[torch.arange(n), ids[1:]] = peak.float()
    x = x.to(TYPES[kind][0]).cuda()
    plan = _plan(rows)
    logp, stats = B.pp_token_logp(plan, x, ids.cuda(), temperature)
    temp = float(np.float32(temperature))
    x64, y = _f64(x)[:n], ids[1:].numpy()
    own = x64[np.arange(n), y]
    others = np.exp((x64 - own[:, None]) / temp)
    others[np.arange(n), y] = 0
    want = -np.log1p(others.sum(1))
    err = np.abs(_f64(logp)[1:] - want)
    assert (err <= U * 8.3 + np.minimum(-want, U * 600)).all(), (err / U).max()
    # the token's own column: g (1 - p) / temperature
    d = B.pp_token_logp_bwd(plan, x, ids.cuda(), logp, stats, torch.ones(n + 1, device="cuda"), temperature)
    got = _f64(d)[np.arange(n), y]
    tol = (U * 8.5 + np.minimum(-want, U * 600)) / temp + TYPES[kind][1] * -want / temp + TYPES[kind][2]
    assert (np.abs(got + np.expm1(want) / temp) <= tol).all()


@pytest.mark.parametrize("T,V,kind", [(9600, 66001, "fp16"), (9601, 33001, "fp32"), (20000, 40000, "fp32")])
def test_blocks_that_look_over_several_rows_of_other_types(T, V, kind):
    from paper_2602_24082_b200 import binding as B
    rows = [[(T - 310, (200, 7))], [(2, (1, 100))]]
    g = torch.Generator(device="cuda").manual_seed(0)
    logits = torch.randn(T, V, generator=g, device="cuda", dtype=TYPES[kind][0])
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    (a, s), (b, _) = (B.pp_token_logp(_plan(rows, desc_on_device=d), logits, ids) for d in (False, True))
    assert torch.equal(a, b)
    r, t = (torch.tensor(x, device="cuda") for x in zip(*P.predictions(rows)))
    x = logits[r].double()
    want = torch.log_softmax(x, -1)[torch.arange(len(t), device="cuda"), ids[t]]
    assert float((a[t].double() - want).abs().max()) < U * (600 + 8 * 12 + 8 * 30)
    used = torch.zeros(T, dtype=torch.bool, device="cuda")
    used[r] = True
    assert not s[~used].any() and torch.equal(s[r, 0].double(), x.amax(1)) and a.count_nonzero() <= len(t)


@pytest.mark.parametrize("n,V,kind,extra", [(129, 300, "bf16", 0), (500, 300, "fp32", 5000), (700, 1000, "fp16", 0), (1500, 40, "bf16", 0),
                                            (1200, 33000, "bf16", 0), (1100, 130001, "fp32", 0), (3000, 1, "fp32", 0), (3000, 7001, "fp32", 4000)])
def test_many_responses_to_a_prompt(n, V, kind, extra):
    """Their first tokens share a row of the gradient; ids that many of them have, some not learned, some beyond the vocabulary."""
    from paper_2602_24082_b200 import binding as B
    rows, T = [[(3 + extra, (1, 2) * (n // 2) + (1,) * (n % 2))]], 3 + extra + n // 2 * 3 + n % 2
    g = torch.Generator(device="cuda").manual_seed(n)
    logits = torch.randn(T, V, generator=g, device="cuda").to(TYPES[kind][0])
    ids = (torch.rand(T, generator=g, device="cuda") ** 3 * V).long()          # (the first ones often)
    ids[torch.rand(T, generator=g, device="cuda") < 0.1] = -1
    plan = _plan(rows)
    logp, stats = B.pp_token_logp(plan, logits, ids)
    grad = torch.randn(T, generator=g, device="cuda")
    d = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, grad)
    r = 2 + extra
    y = torch.tensor([t for row, t in P.predictions(rows) if row == r], device="cuda")
    assert len(y) == n
    y = y[ids[y] >= 0]
    lp = torch.log_softmax(logits[r].double(), 0)
    assert float((logp[y].double() - lp[ids[y]]).abs().max()) < U * (600 + 8 * 12 + 8 * 30)
    w, w_abs = (torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, ids[y], x) for x in (grad[y].double(), grad[y].double().abs()))
    want = w - lp.exp() * grad[y].double().sum()
    # (the sums of the gradients, in 64 bits, are rounded once each: one step of what is subtracted from one another)
    size = w_abs * -torch.expm1(lp) + lp.exp() * float(grad[y].abs().sum())
    _, half, tiny = TYPES[kind]
    err = (d[r].double() - want).abs()
    assert (err <= half * want.abs() * (1 + 2 * half) + U * (700 + 8 * np.log2(V + 1)) * size + tiny).all()
    # ids beyond the vocabulary have no column, and what they write to is nobody's
    ids[y[::2]] += V
    d2 = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, grad)
    z = y[1::2]
    want = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, ids[z], grad[z].double()) - lp.exp() * grad[y].double().sum()
    assert ((d2[r].double() - want).abs() <= half * want.abs() * (1 + 2 * half) + U * (700 + 8 * np.log2(V + 1)) * size + tiny).all()
    assert torch.equal(B.pp_token_logp_bwd(plan, logits, ids, logp, stats, grad, d_logits=logits), d2)


def test_time_of_many_responses_is_not_their_square():
    from paper_2602_24082_b200 import binding as B
    times = []
    for n in (4096, 32768):
        rows = [[(3, (1,) * n)]]
        logits = torch.zeros(n + 3, 500, dtype=torch.bfloat16, device="cuda")
        ids = torch.arange(n + 3, device="cuda") % 500
        plan = _plan(rows)
        logp, stats = B.pp_token_logp(plan, logits, ids)
        grad, took = torch.ones(n + 3, device="cuda"), []
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            B.pp_token_logp_bwd(plan, logits, ids, logp, stats, grad)
            b.record()
            torch.cuda.synchronize()
            took.append(a.elapsed_time(b))
        times.append(min(took))
    assert times[1] < 24 * times[0]        # (8 times as many: 64 times as long, were it the square)
