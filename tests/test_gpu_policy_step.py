"""One policy-training step of a layer on image prompts, all calls in a row as a program makes them, against fp64
autograd on the unpacked sequences (x, y^k): positions with axes, rotary embedding out of a fused
projection's buffer, packed attention, logits, log-probabilities, policy loss, and all the way back into the
projection's gradient.

Tolerance: between the projection's output and its gradient lie the roundings to bf16 of q and k, O, the logits, d logits, dO,
P and dS inside the attention, dQ / dK / dV, and what is rotated back: eight on any path, each half a step, 2^-8 of its
values (2-norm), which add up to 2^-5 at most."""
import numpy as np
import pytest
import torch

from oracle import axes as A
from oracle import policy as P
from paper_2602_24082_b200 import workloads as W

pytestmark = pytest.mark.gpu

ROWS = [[(70, (40, 9, 130)), (21, (30, 1))], [(200, (64, 65, 17))]]
STARTS, GRIDS = [3, 40, 274, 340], [(1, 5, 6), (2, 2, 3), (1, 3, 4), (1, 9, 11)]
SECTIONS, BASE, V = (8, 12, 12), 10000.0, 517
POLICY = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.1, reduction="response", scale=0.125)


def _reference(qkv, w, ids, old, ref, reward, Hq, Hkv, D):
    """(total loss, d qkv) by autograd, sequence by sequence."""
    leaf = qkv.double().cpu().requires_grad_()
    wo, ids = w.double().cpu(), ids.cpu()
    pos = torch.from_numpy(A.position_ids(ROWS, STARTS, GRIDS)).double()
    axis = [a for a, n in enumerate(SECTIONS) for _ in range(n)]
    freq = BASE ** (-2.0 * torch.arange(D // 2, dtype=torch.float64) / D)
    adv = P.advantages(ROWS, reward.cpu(), "normalized")
    total, logps, k = 0, torch.zeros(len(leaf), dtype=torch.float64), 0
    for prompt, resp in P.sequences(ROWS):
        for y in resp:
            at = torch.tensor(list(prompt) + list(y))
            x = leaf[at]
            angle = (pos[axis][:, at].T * freq)[:, None]
            c, s = angle.cos(), angle.sin()
            turn = lambda z: torch.cat([z[..., :D // 2] * c - z[..., D // 2:] * s, z[..., D // 2:] * c + z[..., :D // 2] * s], -1)
            q, key, v = turn(x[:, :Hq]), turn(x[:, Hq:Hq + Hkv]), x[:, Hq + Hkv:]
            rep = lambda z: z.repeat_interleave(Hq // Hkv, 1)
            score = torch.einsum("ihd,jhd->hij", q, rep(key)) * D ** -0.5
            score = score.masked_fill(torch.ones(len(at), len(at)).triu(1).bool(), -torch.inf)
            o = torch.einsum("hij,jhd->ihd", score.softmax(-1), rep(v)).flatten(1)
            lp = torch.log_softmax(o[:-1] @ wo, -1)[torch.arange(len(at) - 1), ids[at[1:]]][len(prompt) - 1:]
            logps[list(y)] = lp.detach()
            if old is not None:
                rho = (lp - old[list(y)]).exp()
                d = ref[list(y)] - lp
                total = total + POLICY["scale"] * (-torch.minimum(rho * adv[k], rho.clamp(0.8, 1.28) * adv[k])
                                                   + 0.1 * (d.exp() - d - 1)).mean()
            k += 1
    if old is None:
        return logps
    total.backward()
    return float(total.detach()), leaf.grad


def test_step_matches_autograd_on_unpacked_sequences():
    from paper_2602_24082_b200 import binding as B
    Hq, Hkv, D = 4, 2, 64
    w = W.Workload("step", ROWS, Hq, Hkv, D, seed=0)
    T, N = w.total_tokens, 8
    g = torch.Generator().manual_seed(0)
    rand = lambda *shape: torch.randn(*shape, generator=g)
    qkv = rand(T, Hq + 2 * Hkv, D).bfloat16().cuda()
    wo = (rand(Hq * D, V) / 8).bfloat16().cuda()
    ids = torch.randint(0, V, (T,), generator=g).cuda()
    reward = rand(N).cuda()
    # ratios of 1, 1.65 and 0.61, away from the borders at 0.8 and 1.28: rounded logits do not move a token across
    lp = _reference(qkv, wo, ids, None, None, reward, Hq, Hkv, D)
    old = (lp - 0.5 * torch.randint(-1, 2, (T,), generator=g)).float()
    ref = (lp + 0.2 * rand(T)).float()
    loss_want, d_want = _reference(qkv, wo, ids, old.double(), ref.double(), reward, Hq, Hkv, D)

    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    plan = B.plan_for(w)
    starts, grids, old, ref = i32(STARTS), i32(GRIDS), old.cuda(), ref.cuda()

    def step():
        pos, status = B.pp_position_ids_axes(plan, starts, grids)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:].contiguous()
        new = lambda h: torch.empty(T, h, D, dtype=torch.bfloat16, device="cuda")
        q, k = B.pp_rope_qk_axes(plan, q, k, pos, SECTIONS, BASE, q_out=new(Hq), k_out=new(Hkv))
        o, lse = B.pp_attn_fwd(plan, q, k, v, D ** -0.5, for_backward=True)
        logits = o.flatten(1) @ wo
        logp, stats = B.pp_token_logp(plan, logits, ids)
        loss, kl, clipped, adv, d_logp = B.pp_policy_loss(plan, logp, old, ref, reward, **POLICY)
        d_logits = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, d_logp, d_logits=logits)
        d_o = (d_logits @ wo.T).view(T, Hq, D)
        dq, dk, dv = B.pp_attn_bwd(plan, q, k, v, o, lse, d_o, D ** -0.5)
        d_qkv = torch.empty_like(qkv)
        B.pp_rope_qk_axes(plan, dq, dk, pos, SECTIONS, BASE, inverse=True, q_out=d_qkv[:, :Hq], k_out=d_qkv[:, Hq:Hq + Hkv])
        d_qkv[:, Hq + Hkv:] = dv
        return loss, logp, d_qkv, status

    loss, logp, d_qkv, status = step()
    torch.cuda.synchronize()
    assert plan.status() == (0, 0) and status.tolist() == [0, 0]
    # (logits of size 2 in bf16: 2^-7 each way, and what O's rounding moves them by)
    resp = [t for _, t in P.predictions(ROWS)]
    assert float((logp.double().cpu() - lp)[resp].abs().max()) < 2.0 ** -4
    assert abs(float(loss.double().sum()) - loss_want) < 2.0 ** -5 * (1 + abs(loss_want))
    err = (d_qkv.double().cpu() - d_want).norm(dim=(0, 2)) / d_want.norm(dim=(0, 2))
    assert float(err.max()) < 2.0 ** -5, err
    # captured and replayed on other projections
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            held = step()
    torch.cuda.synchronize()
    qkv.copy_(qkv.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    again = step()
    assert torch.equal(held[0], again[0]) and torch.equal(held[1], again[1]) and not torch.equal(held[1], logp)
    assert float((held[2].double() - again[2].double()).norm() / again[2].double().norm()) < 2e-3   # (order of dQ's sums)


def test_the_preference_loss_takes_the_same_log_probabilities():
    """pp_token_logp -> pp_preference_loss -> pp_token_logp_bwd, against autograd on the logits."""
    from paper_2602_24082_b200 import binding as B
    w = W.Workload("dpo", ROWS, 4, 2, 64, seed=0)
    T = w.total_tokens
    g = torch.Generator().manual_seed(3)
    logits = torch.randn(T, 300, generator=g).cuda()
    ids = torch.randint(0, 300, (T,), generator=g, dtype=torch.int32).cuda()
    plan = B.plan_for(w)
    logp, stats = B.pp_token_logp(plan, logits, ids)
    ref = logp + 0.1 * torch.randn(T, generator=g).cuda()
    _, _, loss, d_logp = B.pp_preference_loss(plan, logp, ref, 0.1)
    d = B.pp_token_logp_bwd(plan, logits, ids, logp, stats, d_logp)
    leaf = logits.double().requires_grad_()
    r, t = (torch.tensor(x, device="cuda") for x in zip(*P.predictions(ROWS)))
    lp = torch.log_softmax(leaf, -1)[r, ids.long()[t]]
    at, total = 0, 0
    full = torch.zeros(T, dtype=torch.float64, device="cuda").index_put((t,), lp - ref.double()[t])
    for _, resp in P.sequences(ROWS):
        reward = torch.stack([0.1 * full[y[0]:y[-1] + 1].sum() for y in resp])
        pairs = [(a, b) for a in range(len(resp)) for b in range(a)]
        total = total - sum(torch.nn.functional.logsigmoid(reward[a] - reward[b]) for a, b in pairs) / len(pairs)
    total.backward()
    # the loss is within 1e-4 (its own test), its gradient too; the logits' is a sum of products with it
    assert abs(float(loss.double().sum() - total.detach())) < 1e-4 * float(total.detach())
    assert float((d.double() - leaf.grad).norm() / leaf.grad.norm()) < 2e-4


@pytest.mark.parametrize("broken", ["offset", "length", "tokens"])
def test_a_refused_plan_leaves_the_outputs_as_they_were(broken):
    """Descriptors that only the device sees: the plan's status says so, and the calls around it read and write nothing by
    them.  (Offsets that point far outside among them.)"""
    from paper_2602_24082_b200 import binding as B
    rgo, gpl, gro, rl = [np.asarray(a, np.int32) for a in ([0, 1, 2], [5, 7], [0, 2, 3], [4, 3, 6])]
    if broken == "offset":
        gro[1] = 2000000000
    elif broken == "length":
        rl[1] = -2000000000
    else:
        gpl[0] = 6
    plan = B.pp_build_plan((rgo, gpl, gro, rl), 2, 1, 64, 25, desc_on_device=True)
    f = lambda *shape: torch.full(shape, 7.0, device="cuda")
    ids = torch.zeros(25, dtype=torch.int64, device="cuda")
    logp, stats, d = f(25), f(25, 2), f(25, 99)
    B.pp_token_logp(plan, f(25, 99), ids, token_logp=logp, row_stats=stats)
    B.pp_token_logp_bwd(plan, f(25, 99), ids, f(25), f(25, 2), f(25), d_logits=d)
    q, k = f(25, 2, 64).bfloat16(), f(25, 1, 64).bfloat16()
    pos = torch.full((3, 25), 7, dtype=torch.int32, device="cuda")
    B.pp_position_ids_axes(plan, pos[0, :1].contiguous(), pos[:1, :3].contiguous(), out=pos)
    B.pp_rope_qk_axes(plan, q, k, pos, (8, 12, 12))
    B.pp_policy_loss(plan, f(25), f(25), f(25), f(3))
    torch.cuda.synchronize()
    assert plan.status()[0] in (1, 2)
    assert all((x == 7).all() for x in (logp, stats, d, q, k, pos))


def test_calls_of_two_streams_on_one_plan():
    """None of the calls around the attention changes the plan: they may run at the same time."""
    from paper_2602_24082_b200 import binding as B
    w = W.Workload("two", [[(300, (200, 100))], [(500, (40, 300, 77))]] * 4, 8, 2, 64, seed=0)
    T = w.total_tokens
    plan = B.plan_for(w)
    g = torch.Generator(device="cuda").manual_seed(0)
    data = []
    for _ in range(2):
        logits = torch.randn(T, 5000, generator=g, device="cuda")
        data.append((logits, torch.randint(0, 5000, (T,), generator=g, device="cuda"), torch.randn(20, generator=g, device="cuda")))

    def work(logits, ids, reward):
        logp, stats = B.pp_token_logp(plan, logits, ids)
        loss, _, _, _, d_logp = B.pp_policy_loss(plan, logp, None, None, reward, kl_coef=0.1)
        return loss, B.pp_token_logp_bwd(plan, logits, ids, logp, stats, d_logp)

    want = [work(*x) for x in data]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in data]
    got = [None, None]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = work(*data[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))


@pytest.mark.parametrize("prompts,responses", [((5, 7), (4, 3, 6)), ((900, 800), (700, 650, 900)), ((3000, 2000), (2100, 1700, 1800))],
                         ids=["warps", "four_blocks", "eight_blocks"])
def test_a_refused_plan_leaves_every_output_as_it_was(prompts, responses):
    """All outputs given, through the C entries, for segments that a warp, a block and clusters of blocks take."""
    import ctypes
    from paper_2602_24082_b200 import binding as B
    T, V = sum(prompts) + sum(responses), 99
    desc = [np.asarray(a, np.int32) for a in ([0, 1, 2], (prompts[0] + 1,) + prompts[1:], [0, 2, 3], responses)]
    plan = B.pp_build_plan(tuple(desc), 2, 1, 64, T, desc_on_device=True)
    f = lambda *shape: torch.full(shape, 7.0, device="cuda")
    i = lambda *shape: torch.full(shape, 7, dtype=torch.int32, device="cuda")
    x, t, ids, status, pos = f(T, V), f(T), torch.zeros(T, dtype=torch.int64, device="cuda"), i(2), i(3, T)
    start, grid = i(1), i(1, 3)
    logp, stats, d, grad = f(T), f(T, 2), f(T, V), f(T)
    adv, loss, kl, cut = f(3), f(3), f(3), f(3)
    q, k = f(T, 2, 64).bfloat16(), f(T, 1, 64).bfloat16()

    class Policy(ctypes.Structure):
        _fields_ = [("mode", ctypes.c_int32), ("reduction", ctypes.c_int32)] + [(n, ctypes.c_double) for n in "abcde"]

    L, h, p, s = B.lib(), plan.handle, (lambda a: a.data_ptr()), torch.cuda.current_stream().cuda_stream
    axis = ctypes.create_string_buffer(bytes(32), 32)
    policy = Policy(2, 0, 0.2, 0.2, 0.1, 1.0, 1e-6)
    mask = torch.ones(T, dtype=torch.bool, device="cuda")
    assert L.pp_token_logp(h, p(x), 2, V, V, p(ids), 1, 1.0, p(logp), p(stats), s) == 0
    assert L.pp_token_logp_bwd(h, p(x), 2, V, V, p(ids), 1, 1.0, p(t), p(stats), p(t), p(d), V, s) == 0
    assert L.pp_policy_loss(h, ctypes.byref(policy), p(t), p(t), p(t), p(t), p(mask), p(adv), p(loss), p(kl), p(cut), p(grad), s) == 0
    assert L.pp_position_ids_axes(h, 1, p(start), p(grid), p(pos), p(status), s) == 0
    assert L.pp_rope_qk_axes(h, p(q), 128, p(k), 64, p(q), 128, p(k), 64, p(pos), 3, axis, 10000.0, 0, s) == 0
    torch.cuda.synchronize()
    assert plan.status()[0] in (1, 2)
    for out in (x, t, logp, stats, d, adv, loss, kl, cut, grad, status, pos, q, k):
        assert (out == 7).all()
