"""GPU parity of the clipped policy loss against the fp64 oracle.

Everything is computed in 64 bits and rounded to fp32 once (u = 2^-24); exp, expm1 and the sums of a few thousand
terms in another order are off by less than 2^-40 of the terms' magnitudes.  exp(d) - d - 1 loses to
cancellation what d^2 / 2 is smaller than d: 2^-52 d, which 2^-40 covers for the magnitudes it is compared at."""
import numpy as np
import pytest
import torch

from oracle import policy as P
from paper_2602_24082_b200 import workloads as W

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ROUND = 2.0 ** -40

CASES = {
    "pair": [[(64, (32, 48))]],
    "ragged": [[(257, (5, 128, 31))], [(1, (1, 300))]],
    "single": [[(97, (64,)), (128, (128, 128, 7, 9, 40))], [(700, (1, 1))]],
    "ones": [[(1, (1,) * 37)] for _ in range(9)],
    "one_token": [[(1, (1,))]],
    "team2": [[(100, (90, 120, 1, 70) * 5)]],
    "team4": [[(150, (140, 250, 201))], [(1, (299,))]],
    "team8": [[(400, (511, 289, 400))], [(1, (799,))]] * 40,
    "parts2": [[(900, (1023, 1, 577))]],
    "parts4": [[(2000, (2047, 1, 2577))]],
    "parts8": [[(5000, (4097, 6000, 4100))]],
    "long": [[(9, (9000, 8191))], [(12000, (7000,))]],
    "many": [[(3, (40, 2)), (1, (1,) * 33)]] * 150,
    "groups": [[(2, (3, 1)), (1, (1,))]] * 1100,
    "mean20": [[(20, (25, 15, 21)), (9, (40,))]] * 9,
    "mean40": [[(40, (45, 30, 51)), (9, (80,))]] * 9,
}


def _inputs(rows, mode, seed, masked):
    rng = np.random.default_rng(seed)
    T = sum(p + sum(rs) for row in rows for p, rs in row)
    N = sum(len(rs) for row in rows for _, rs in row)
    lp = -rng.gamma(1.0, 1.5, T)
    old, ref = lp + np.where(rng.random(T) < 0.2, 0.5, 0.02) * rng.normal(size=T), lp + 0.1 * rng.normal(size=T)
    reward = rng.normal(size=T if mode == "token" else N)
    mask = None
    if masked:
        mask = rng.random(T) < 0.7
        y = P.sequences(rows)[0][1][-1]
        mask[y[0]:y[-1] + 1] = False           # a response with nothing left
    f = lambda x: x.astype(np.float32)
    return f(lp), f(old), f(ref), f(reward), mask


def _cuda(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _check(got, want):
    loss, kl, cut, adv, grad = [None if x is None else x.double().cpu().numpy() for x in got]
    for a, b in ((loss, want[0]), (kl, want[1]), (cut, want[2]), (adv, want[3]), (grad, want[4])):
        assert (a is None) == (b is None)
        if a is not None:
            size = np.abs(b[np.isfinite(b)]).max(initial=0)
            assert np.array_equal(np.isfinite(a), np.isfinite(b))
            fine = np.isfinite(b)
            assert (np.abs(a - b)[fine] <= (U * np.abs(b) + ROUND * (size + 1e-30))[fine] + 2.0 ** -149).all()


@pytest.mark.parametrize("rows", list(CASES.values()), ids=list(CASES))
@pytest.mark.parametrize("mode", ["given", "centered", "normalized", "token"])
@pytest.mark.parametrize("reduction,masked", [("response", False), ("token", True), ("response", True)])
def test_parity(rows, mode, reduction, masked):
    from paper_2602_24082_b200 import binding as B
    lp, old, ref, reward, mask = _inputs(rows, mode, 3, masked)
    if mode != "token":
        reward[0] = 0.0
    kw = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.04, reduction=reduction, scale=0.3)
    want = P.policy_loss(rows, lp, old, ref, reward, mode=mode, mask=mask, **kw)
    plan = B.plan_for(W.Workload("policy", rows, 2, 1, 64, seed=0), desc_on_device=masked)
    # prompt and masked entries may hold anything
    hidden = np.ones(len(lp), bool)
    for _, resp in P.sequences(rows):
        for y in resp:
            hidden[y[0]:y[-1] + 1] = False if mask is None else ~mask[y[0]:y[-1] + 1]
    for x in (lp, old, ref) + ((reward,) if mode == "token" else ()):
        x[hidden] = [np.nan, np.inf, -np.inf][len(rows) % 3]
    got = B.pp_policy_loss(plan, _cuda(lp), _cuda(old), _cuda(ref), _cuda(reward), advantage=mode, token_mask=_cuda(mask), **kw)
    again = B.pp_policy_loss(plan, _cuda(lp), _cuda(old), _cuda(ref), _cuda(reward), advantage=mode, token_mask=_cuda(mask), **kw)
    torch.cuda.synchronize()
    assert plan.status() == (0, 0)
    _check(got, want)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(got, again))
    assert not got[4].cpu().numpy()[hidden].any()


@pytest.mark.parametrize("rows", [CASES["ragged"], CASES["parts4"]], ids=["ragged", "parts4"])
def test_without_old_reference_or_gradient(rows):
    from paper_2602_24082_b200 import binding as B
    lp, old, ref, reward, _ = _inputs(rows, "given", 4, False)
    plan = B.plan_for(W.Workload("policy", rows, 2, 1, 64, seed=0))
    for o, r in ((None, None), (old, None), (None, ref)):
        want = P.policy_loss(rows, lp, o, r, reward, mode="given", kl_coef=0.1)
        args = (plan, _cuda(lp), _cuda(o), _cuda(r), _cuda(reward))
        _check(B.pp_policy_loss(*args, advantage="given", kl_coef=0.1), want)
        none = B.pp_policy_loss(*args, advantage="given", kl_coef=0.1, want_grad=False)
        assert none[4] is None
        _check(none, want[:4] + (None,))


def test_borders_and_extremes():
    """Ratios exactly at a border keep their gradient (the smaller of two equal terms); beyond it only the
    side that the advantage pulls away from; ratios that overflow fp32."""
    from paper_2602_24082_b200 import binding as B
    rows = [[(2, (8,))]]
    plan = B.plan_for(W.Workload("policy", rows, 2, 1, 64, seed=0))
    f = lambda *x: torch.tensor(x, device="cuda")
    lp = torch.zeros(10, device="cuda")
    old = f(0, 0, 0, -np.log(2), np.log(2), -np.log(4), np.log(4), -200, 200, float("nan")).float()
    rho = np.exp(-old.double().cpu().numpy())[2:]
    for A in (1.0, -1.0, 0.0):
        loss, _, cut, adv, grad = B.pp_policy_loss(plan, lp, old, None, f(A), advantage="given", reduction="token",
                                                   token_mask=f(*[True] * 9 + [False]), clip_low=0.5, clip_high=1.0)
        want = np.zeros(8)
        clip = np.clip(rho, 0.5, 2.0)
        keep = rho * A <= clip * A
        want[keep] = -(rho * A)[keep]
        want[7] = 0
        with np.errstate(over="ignore"):
            assert np.allclose(grad.cpu().numpy()[2:], want.astype(np.float32), rtol=2e-7, atol=0)
        assert float(cut[0]) == np.float32((~keep[:7]).sum() / 7)


@pytest.mark.parametrize("mode", ["centered", "normalized"])
def test_equal_rewards_have_no_advantage(mode):
    """Their mean is the reward itself, exactly, whatever it and their number are."""
    from paper_2602_24082_b200 import binding as B
    sizes = [1, 2, 3, 5, 6, 7, 11, 33, 49, 100, 641]
    rows = [[(2, (1,) * n)] for n in sizes]
    plan = B.plan_for(W.Workload("policy", rows, 2, 1, 64, seed=0))
    rng = np.random.default_rng(0)
    lp = _cuda(-rng.gamma(1.0, 1.5, sum(sizes) + 2 * len(sizes)).astype(np.float32))
    for _ in range(20):
        r = np.repeat(rng.normal(size=len(sizes)).astype(np.float32), sizes)
        loss, _, _, adv, grad = B.pp_policy_loss(plan, lp, None, None, _cuda(r), advantage=mode)
        assert not adv.any() and not loss.any() and not grad.any()


def test_gradient_against_differences():
    """fp32 losses of size 1 moved by 2^-9 along a direction: 2 u / h of rounding and the curvature's h^2.  Ratios
    stay clear of the borders, where there is no slope."""
    from paper_2602_24082_b200 import binding as B
    rows = [[(5, (20, 7))], [(3, (11, 9, 1))]]
    lp, old, ref, reward, _ = _inputs(rows, "normalized", 6, False)
    ratio = np.exp(lp.astype(np.float64) - old)
    old = np.where(np.abs(ratio - 0.8) + 0 < 0.05, lp, np.where(np.abs(ratio - 1.2) < 0.05, lp, old)).astype(np.float32)
    plan = B.plan_for(W.Workload("policy", rows, 2, 1, 64, seed=0))
    call = lambda x: B.pp_policy_loss(plan, x, _cuda(old), _cuda(ref), _cuda(reward), kl_coef=0.1, scale=0.2)
    grad = call(_cuda(lp))[4].double()
    h = 2.0 ** -9
    for seed in range(4):
        v = torch.sign(torch.randn(len(lp), generator=torch.Generator().manual_seed(seed))).cuda()
        up, down = (call(_cuda(lp) + s * h * v)[0].double().sum() for s in (1, -1))
        # (lp of size 8 moves by h up to 2^-21)
        assert abs(float((up - down) / (2 * h) - (grad * v).sum())) < float(grad.abs().sum()) * (2.0 ** -21 / h + 4 * h * h) + 8 * U / h


def test_streams_and_graphs():
    from paper_2602_24082_b200 import binding as B
    rows = CASES["parts2"] + CASES["ragged"]
    lp, old, ref, reward, mask = (_cuda(x) for x in _inputs(rows, "normalized", 7, True))
    plan = B.plan_for(W.Workload("policy", rows, 2, 1, 64, seed=0))
    step = lambda: B.pp_policy_loss(plan, lp, old, ref, reward, token_mask=mask, kl_coef=0.1)
    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        there = step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            held = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(there, want))
    reward.copy_(torch.roll(reward, 1))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, step()))
    assert not torch.equal(held[0], want[0])


def test_refusals():
    from paper_2602_24082_b200 import binding as B
    rows = [[(3, (4, 2))]]
    plan = B.plan_for(W.Workload("policy", rows, 2, 1, 64, seed=0))
    lp, r = torch.zeros(9, device="cuda"), torch.zeros(2, device="cuda")
    for args in ((lp[:8], None, None, r), (lp, lp.double(), None, r), (lp, None, lp.cpu(), r), (lp, None, None, lp)):
        with pytest.raises(ValueError):
            B.pp_policy_loss(plan, *args)
    for kw in (dict(advantage="rank"), dict(reduction="mean"), dict(advantage="token"),
               dict(token_mask=torch.ones(9, device="cuda")), dict(token_mask=torch.ones(8, device="cuda").bool())):
        with pytest.raises(ValueError):
            B.pp_policy_loss(plan, lp, None, None, r, **kw)
    nan = float("nan")
    for kw in (dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_low=nan), dict(clip_high=-1), dict(clip_high=nan),
               dict(kl_coef=-1), dict(kl_coef=nan), dict(scale=nan), dict(eps=0), dict(eps=nan)):
        with pytest.raises(B.PPError):
            B.pp_policy_loss(plan, lp, None, None, r, **kw)


@pytest.mark.parametrize("mode,reduction,masked", [("normalized", "response", True), ("token", "token", False)])
@pytest.mark.parametrize("rows", [[[(9, (2000,) * 80)]], [[(9, (500,) * 160)]], [[(9, (700,) * 40)]]],
                         ids=["four_blocks_of_eight", "one_block_of_four", "four_blocks"])
def test_parity_where_clusters_would_not_fit_the_chip(rows, mode, reduction, masked):
    """Long responses, many of them: four blocks for each where eight would be more than four to an SM, and one where
    four would be."""
    from paper_2602_24082_b200 import binding as B
    lp, old, ref, reward, mask = _inputs(rows, mode, 5, masked)
    kw = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.04, reduction=reduction, scale=0.3)
    want = P.policy_loss(rows, lp, old, ref, reward, mode=mode, mask=mask, **kw)
    plan = B.plan_for(W.Workload("policy", rows, 2, 1, 64, seed=0))
    args = (plan, _cuda(lp), _cuda(old), _cuda(ref), _cuda(reward))
    got = B.pp_policy_loss(*args, advantage=mode, token_mask=_cuda(mask), **kw)
    _check(got, want)
    again = B.pp_policy_loss(*args, advantage=mode, token_mask=_cuda(mask), **kw)
    assert plan.status() == (0, 0) and all(a is b is None or torch.equal(a, b) for a, b in zip(got, again))
