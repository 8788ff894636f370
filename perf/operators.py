"""The steps of a policy-training step around packed attention, as measurable cases.

A case is a dict of plain values.  `op` names the operator:

  logp       log-probabilities of the packed tokens from the logits
  logp_bwd   the gradient of the logits, given that of the log-probabilities
  policy     clipped policy loss with a KL term over the responses, with its gradient
  positions  position ids with a time, a height and a width axis, from the images' grids
  rope       rotary embedding of Q and K with these positions, or its inverse (the backward pass)

Rows are packed as [prompt | response 1 | ... | response n]; `layout` seeds the lengths, so a case
always means the same structure while the tensors follow the caller's seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---------------------------------------------------------------------------- structures

def _groups(case):
    """[(prompt length, (response lengths, ...)), ...]"""
    rng = np.random.Generator(np.random.PCG64(case["layout"]))
    if case["shape"] == "sample":
        return [(64, (32, 48))]
    if case["shape"] == "pairs":
        return [(int(np.clip(round(512 * math.exp(0.5 * rng.standard_normal())), 64, 2048)),
                 tuple(int(rng.integers(64, 513)) for _ in range(2))) for _ in range(8)]
    # "drawn": groups of about `mean` tokens, `n` responses each, prompt : mean response = `rho`
    groups, left, n, rho = [], case["tokens"], case["n"], case["rho"]
    while left > 0:
        total = int(min(16384, max(n + 1, round(case["mean"] * math.exp(0.5 * rng.standard_normal())))))
        total = max(n + 1, min(total, left))
        rs = [max(1, int(round(total / (rho + n) * rng.uniform(0.5, 1.5)))) for _ in range(n)]
        while sum(rs) >= total:
            rs[int(np.argmax(rs))] -= 1
        groups.append((total - sum(rs), tuple(rs)))
        left -= total
    return groups


def _segments(groups):
    """(start, length, group, 0 for the prompt or the response's number from 1 on) of every segment"""
    out, t = [], 0
    for g, (p, rs) in enumerate(groups):
        out.append((t, p, g, 0))
        t += p
        for k, r in enumerate(rs):
            out.append((t, r, g, k + 1))
            t += r
    return out


def _tokens(groups):
    return sum(p + sum(rs) for p, rs in groups)


def _predicted(groups):
    """(tokens, rows): the response tokens, and per token the row whose logits predict it -- the token
    before it, and the prompt's last for the first of every response."""
    tok, row, prompt_end = [], [], 0
    for a, n, _, k in _segments(groups):
        if k == 0:
            prompt_end = a + n
            continue
        t = np.arange(a, a + n)
        r = t - 1
        r[0] = prompt_end - 1
        tok.append(t)
        row.append(r)
    return np.concatenate(tok), np.concatenate(row)


def _spans(case, groups, seed=0):
    """Images and videos in the prompts: (first token, (frames, height, width)), in token order."""
    rng = np.random.Generator(np.random.PCG64([case["layout"], seed]))
    starts, grids, t = [], [], 0
    for p, rs in groups:
        at = t + int(rng.integers(1, 40))
        side = max(2, min(case["side"], math.isqrt(p // 3)))
        for _ in range(case["images"]):
            h, w = int(rng.integers(2, side + 1)), int(rng.integers(2, side + 1))
            f = int(rng.integers(2, 9)) if rng.random() < 0.2 else 1
            if at + f * h * w >= t + p:
                break
            starts.append(at)
            grids.append((f, h, w))
            at += f * h * w + int(rng.integers(0, 60))
        t += p + sum(rs)
    return np.asarray(starts, np.int32), np.asarray(grids, np.int32).reshape(-1, 3)


# ---------------------------------------------------------------------------- the cases

def _drawn(tokens, mean, n, rho):
    return {"shape": "drawn", "tokens": tokens, "mean": mean, "n": n, "rho": rho}


def listed():
    return [
        # one short sample: the smallest call, where launches and the split of a row count
        {"name": "logp_tiny", "op": "logp", "shape": "sample", "layout": 0, "vocab": 32000, "type": "bf16",
         "temperature": 1.0, "banned": 0, "ignored": 0.0},
        # the ordinary step of pairwise data on an 8B-class shape
        {"name": "logp_pairs", "op": "logp", "shape": "pairs", "layout": 1, "vocab": 128256, "type": "bf16",
         "temperature": 1.0, "banned": 0, "ignored": 0.0},
        # fp32 logits of an odd vocabulary sampled at a temperature, ids that may not be sampled at -inf, some
        # tokens (tool output) that are not learned
        dict({"name": "logp_odd", "op": "logp", "layout": 2, "vocab": 50257, "type": "fp32", "temperature": 0.7,
              "banned": 19, "ignored": 0.05}, **_drawn(3001, 700, 4, 2)),
        # its backward pass, the ordinary step
        {"name": "logp_bwd_pairs", "op": "logp_bwd", "shape": "pairs", "layout": 1, "vocab": 128256, "type": "bf16",
         "temperature": 1.0, "banned": 0, "ignored": 0.0},
        # fp16 with a scaled loss, an odd vocabulary, many short responses to a prompt
        dict({"name": "logp_bwd_odd", "op": "logp_bwd", "layout": 3, "vocab": 50257, "type": "fp16",
              "temperature": 0.7, "banned": 19, "ignored": 0.05}, **_drawn(2999, 500, 8, 1)),
        # the smallest policy loss: one pair
        {"name": "policy_tiny", "op": "policy", "shape": "sample", "layout": 0, "advantage": "given",
         "reduction": "response", "old": True, "ref": False, "masked": 0.0},
        # long rows, four ranked responses to a prompt, everything on
        dict({"name": "policy_long", "op": "policy", "layout": 4, "advantage": "normalized", "reduction": "response",
              "old": True, "ref": True, "masked": 0.1}, **_drawn(65536, 4096, 4, 4)),
        # a large batch of short answers, sums over tokens
        dict({"name": "policy_many", "op": "policy", "layout": 5, "advantage": "normalized", "reduction": "token",
              "old": True, "ref": True, "masked": 0.1}, **_drawn(40000, 150, 8, 0.5)),
        # position ids of a few image prompts
        dict({"name": "positions_short", "op": "positions", "layout": 6, "images": 2, "side": 24}, **_drawn(5000, 1500, 2, 4)),
        # ... and of long rows with several images and videos in a prompt
        dict({"name": "positions_long", "op": "positions", "layout": 7, "images": 12, "side": 24}, **_drawn(65536, 4096, 2, 16)),
        # one layer of a small batch, head_dim 64, backward: dQ and dK into the buffer of the fused projection
        dict({"name": "rope_short", "op": "rope", "layout": 8, "images": 2, "side": 24, "hq": 14, "hkv": 2, "d": 64,
              "inverse": True, "interleaved": False, "base": 1000000.0}, **_drawn(1999, 1500, 2, 4)),
        # one layer of long rows, forward: Q and K out of the buffer of the fused projection
        dict({"name": "rope_long", "op": "rope", "layout": 7, "images": 12, "side": 24, "hq": 32, "hkv": 8, "d": 128,
              "inverse": False, "interleaved": False, "base": 500000.0}, **_drawn(65536, 4096, 2, 16)),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    op = rng.choice(["logp", "logp", "logp_bwd", "logp_bwd", "policy", "policy", "positions", "rope", "rope"])
    case = dict({"op": op, "layout": rng.randrange(1 << 30)},
                **_drawn(0, log(30, 8000), rng.choice([1, 2, 2, 3, 4, 8, 16]), rng.choice([0.25, 1, 2, 4, 16])))
    if op in ("logp", "logp_bwd"):
        case.update(vocab=log(500, 160000), type=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                    temperature=rng.choice([1.0, 1.0, 0.7, 1.3]), banned=rng.choice([0, 0, 19]),
                    ignored=rng.choice([0.0, 0.0, 0.05]))
        most = 600000000 // (2 if case["type"] == "fp32" else 1)
        case["tokens"] = log(50, min(65536, most // case["vocab"]))
    elif op == "policy":
        case.update(tokens=log(100, 65536), advantage=rng.choice(["given", "centered", "normalized", "normalized", "token"]),
                    reduction=rng.choice(["response", "token"]), old=rng.random() < 0.8, ref=rng.random() < 0.7,
                    masked=rng.choice([0.0, 0.1, 0.5]))
        case["ref"] |= case["n"] == 1      # (a single answer has no advantage over others)
    elif op == "positions":
        case.update(tokens=log(1000, 65536), mean=log(300, 8000), n=rng.choice([1, 2, 2, 4]), rho=rng.choice([1, 2, 4, 16]),
                    images=rng.choice([1, 2, 12]), side=rng.choice([4, 16, 32]))
    else:
        case.update(tokens=log(100, 65536), images=rng.choice([0, 1, 2, 12]), side=rng.choice([4, 16, 32]))
        hkv = rng.choice([1, 2, 4, 8])
        hq = hkv * rng.choice([1, 2, 4, 7, 8])
        case["tokens"] = min(case["tokens"], 2600000 // (hq + hkv))
        case.update(hq=hq, hkv=hkv, d=rng.choice([64, 96, 128, 128]), inverse=rng.random() < 0.5,
                    interleaved=rng.random() < 0.3, base=rng.choice([10000.0, 500000.0, 1000000.0]))
    case["mean"] = max(case["mean"], case["n"] + 1)
    return case


# ---------------------------------------------------------------------------- preparation

def _sections(d):
    """How many of the d / 2 frequencies go by time, height and width."""
    return {64: (8, 12, 12), 96: (12, 18, 18), 128: (16, 24, 24)}[d]


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, generator=gen, device=dev)
    uniform = lambda *shape: torch.rand(*shape, generator=gen, device=dev)
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)
    groups = _groups(case)
    T, N, op = _tokens(groups), sum(len(rs) for _, rs in groups), case["op"]
    st = {"case": case}
    # what a program keeps for a packed batch: the plan, or the index tensors that stand for it in the plain form
    segs = _segments(groups)
    if own:
        from paper_2602_24082_b200 import binding
        off = np.concatenate([[0], np.cumsum([len(rs) for _, rs in groups])])
        desc = (np.arange(len(groups) + 1), np.asarray([p for p, _ in groups]), off,
                np.concatenate([rs for _, rs in groups]))
        st["plan"] = binding.pp_build_plan([a.astype(np.int32) for a in desc], case.get("hq", 32), case.get("hkv", 8),
                                           case.get("d", 128), T)
    tok, row = _predicted(groups)
    st["tok"], st["row"], st["T"], st["N"] = put(tok), put(row), T, N
    rows, at = np.unique(row, return_inverse=True)
    st["rows"], st["at"] = put(rows), put(at)       # the rows that predict something, and which of them predicts a token
    if op in ("logp", "logp_bwd"):
        V = case["vocab"]
        ids = torch.randint(0, V - case["banned"], (T,), generator=gen, device=dev)
        logits = torch.randn(T, V, generator=gen, device=dev, dtype=TYPES[case["type"]])
        logits *= 2.5
        # sampled tokens are mostly likely ones
        logits.index_put_((st["row"], ids[st["tok"]]), (15 * uniform(len(tok))).to(logits.dtype), accumulate=True)
        if case["banned"]:
            logits[:, V - case["banned"]:] = -math.inf
        ids[uniform(T) < case["ignored"]] = -100
        st.update(logits=logits, ids=ids)
        if op == "logp_bwd":
            # what the forward pass left, and the gradient that the loss gave
            logp = torch.zeros(T, device=dev)
            x = logits.float() / case["temperature"]
            m = x.amax(1)
            stats = torch.stack([m, (x - m[:, None]).exp_().sum(1).log()], 1)
            del x
            r, y = st["row"], ids[st["tok"]]
            z = (logits[r, y.clamp(min=0)].float() / case["temperature"] - stats[r, 0]) - stats[r, 1]
            logp[st["tok"]] = torch.where(y >= 0, z, torch.zeros_like(z))
            st.update(logp=logp, stats=stats, grad=rand(T))
    elif op == "policy":
        resp = np.full(T, -1, np.int64)
        grp = []
        for a, n, g, k in segs:
            if k:
                resp[a:a + n] = len(grp)
                grp.append(g)
        st.update(resp=put(resp[resp >= 0]), grp=put(np.asarray(grp)), G=len(groups))
        logp = -1.5 * torch.empty(T, device=dev).exponential_(generator=gen)
        st["logp"] = logp
        # most tokens have hardly moved since they were sampled, some have left the trust region
        st["old"] = logp + torch.where(uniform(T) < 0.1, 0.4, 0.03) * rand(T) if case["old"] else None
        st["ref"] = logp + 0.1 * rand(T) if case["ref"] else None
        st["mask"] = uniform(T) >= case["masked"] if case["masked"] else None
        if case["advantage"] in ("token", "given"):
            st["reward"] = rand(T if case["advantage"] == "token" else N)
        else:
            # right or wrong, in two of three groups with a bonus: in the others all answers may be the same
            st["reward"] = (uniform(N) < 0.4).float() + torch.where(st["grp"] % 3 < 2, 0.1 * rand(N), torch.zeros(N, device=dev))
        st["scale"] = 1.0 / N if case["reduction"] == "response" else 1.0 / len(tok)
    else:
        # (positions follow from the images alone: another batch has others)
        starts, grids = _spans(case, groups, seed if op == "positions" else 0)
        st.update(starts=put(starts), grids=put(grids), seg_of=put(np.repeat(np.arange(len(segs)), [n for _, n, _, _ in segs])),
                  seg_start=put(np.asarray([a for a, _, _, _ in segs])),
                  prompt=put(np.asarray([i - k for i, (_, _, _, k) in enumerate(segs)])),
                  is_resp=put(np.asarray([k > 0 for _, _, _, k in segs])))
        if op == "rope":
            Hq, Hkv, D = case["hq"], case["hkv"], case["d"]
            st["pos"] = _positions(st)
            qkv = rand(T, Hq + 2 * Hkv, D).bfloat16()
            st["q"], st["k"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]
            if case["inverse"]:   # gradients as the attention's backward pass leaves them
                st["q"], st["k"] = st["q"].contiguous(), st["k"].contiguous()
            st["sections"] = _sections(D)
    return st


# ---------------------------------------------------------------------------- one pass

def _scaled(st):
    x = st["logits"][st["rows"]].float()
    return x if st["case"]["temperature"] == 1.0 else x / st["case"]["temperature"]


def _logp(st):
    x, at, y = _scaled(st), st["at"], st["ids"][st["tok"]]
    m = x.amax(1)
    lsum = (x - m[:, None]).exp().sum(1).log()
    z = (x[at, y.clamp(min=0)] - m[at]) - lsum[at]
    logp = torch.zeros(st["T"], device=x.device)
    logp[st["tok"]] = torch.where(y >= 0, z, torch.zeros_like(z))
    # rows that predict nothing have no statistics
    used = torch.zeros(len(m), device=x.device).index_add_(0, at, (y >= 0).float()) > 0
    stats = torch.zeros(st["T"], 2, device=x.device)
    stats[st["rows"]] = torch.where(used[:, None], torch.stack([m, lsum], 1), torch.zeros_like(m)[:, None])
    return {"logp": logp, "stats": stats}


def _logp_bwd(st):
    rows, at, y = st["rows"], st["at"], st["ids"][st["tok"]]
    g = torch.where(y >= 0, st["grad"][st["tok"]], torch.zeros((), device=at.device))
    total = torch.zeros(len(rows), device=at.device).index_add_(0, at, g)
    p = (_scaled(st) - st["stats"][rows, 0:1] - st["stats"][rows, 1:2]).exp()
    d = -total[:, None] * p
    d.index_put_((at, y.clamp(min=0)), g, accumulate=True)
    out = torch.zeros(st["logits"].shape, dtype=st["logits"].dtype, device=at.device)
    out[rows] = (d / st["case"]["temperature"]).to(out.dtype)
    return out


def _policy(st):
    c, tok, resp = st["case"], st["tok"], st["resp"]
    dev, N = tok.device, st["N"]
    zeros = lambda n: torch.zeros(n, dtype=torch.float64, device=dev)
    lp = st["logp"][tok].double()
    old = lp if st["old"] is None else st["old"][tok].double()
    m = torch.ones(len(tok), dtype=torch.bool, device=dev) if st["mask"] is None else st["mask"][tok]
    r = st["reward"].double()
    adv = r
    if c["advantage"] in ("centered", "normalized"):
        count = zeros(st["G"]).index_add_(0, st["grp"], torch.ones_like(r))
        adv = r - (zeros(st["G"]).index_add_(0, st["grp"], r) / count)[st["grp"]]
        if c["advantage"] == "normalized":
            var = zeros(st["G"]).index_add_(0, st["grp"], adv * adv) / (count - 1).clamp(min=1)
            adv = adv / (var.sqrt()[st["grp"]] + 1e-6)
    A = adv[tok] if c["advantage"] == "token" else adv[resp]
    n = zeros(N).index_add_(0, resp, m.double())
    rho = (lp - old).exp()
    u, v = rho * A, rho.clamp(0.8, 1.28) * A
    loss, dlp = -torch.minimum(u, v), torch.where(u <= v, -u, torch.zeros_like(u))
    kl = torch.zeros_like(lp)
    if st["ref"] is not None:
        delta = st["ref"][tok].double() - lp
        kl = torch.expm1(delta) - delta
        loss, dlp = loss + 0.04 * kl, dlp - 0.04 * torch.expm1(delta)
    per = lambda x: zeros(N).index_add_(0, resp, torch.where(m, x, torch.zeros_like(x)))
    inv = torch.where(n > 0, 1 / n, torch.zeros_like(n))
    w = st["scale"] * (inv if c["reduction"] == "response" else torch.ones_like(n))
    grad = zeros(st["T"])
    grad[tok] = torch.where(m, w[resp] * dlp, torch.zeros_like(dlp))
    out = {"loss": w * per(loss), "kl": inv * per(kl), "clipped": inv * per((v < u).double()), "grad": grad}
    if c["advantage"] != "token":
        out["advantage"] = adv
    return {k: x.float() for k, x in out.items()}


def _positions(st):
    T, dev = st["T"], st["seg_of"].device
    t = torch.arange(T, device=dev)
    seg = st["seg_of"]
    prompt = st["prompt"][seg]
    start = st["starts"].long()
    g = st["grids"].long()
    size = g.prod(1)
    saved = torch.zeros(len(start) + 1, dtype=torch.int64, device=dev)   # by how much the spans before are shorter than their tokens
    saved[1:] = (size - g.amax(1)).cumsum(0)
    before = torch.searchsorted(start, t)                # spans that begin in front of t
    at_or_before = torch.searchsorted(start, t, right=True)
    first = lambda x: torch.searchsorted(start, x)
    i = (at_or_before - 1).clamp(min=0)
    inside = torch.zeros_like(t, dtype=torch.bool)
    k = torch.zeros_like(t)
    if len(start):
        k = t - start[i]
        inside = (at_or_before > 0) & (k < size[i])
    base = torch.where(inside, start[i] if len(start) else t, t)
    done = torch.where(inside, i, before)
    seg_start, prompt_start = st["seg_start"][seg], st["seg_start"][prompt]
    resp = st["is_resp"][seg]
    prompt_end = st["seg_start"][prompt + 1 - (~resp).long()]   # (of a prompt token: its own start, not used)
    number = base - seg_start - (saved[done] - saved[first(seg_start)])
    behind = (prompt_end - prompt_start) - (saved[first(prompt_end)] - saved[first(prompt_start)])
    number = number + torch.where(resp, behind, torch.zeros_like(behind))
    if not len(start):
        return number.to(torch.int32).expand(3, T).contiguous()
    h, w = g[i, 1], g[i, 2]
    zero = torch.zeros_like(k)
    axes = [torch.where(inside, x, zero) for x in (k // (h * w), k // w % h, k % w)]
    return torch.stack([number + x for x in axes]).to(torch.int32)


def _axis_of(c, dev):
    s = _sections(c["d"])
    if not c["interleaved"]:
        return torch.repeat_interleave(torch.arange(3, device=dev), torch.tensor(s, device=dev))
    # in turns, an axis dropping out when it has had its share
    i = torch.arange(sum(s), device=dev)
    turn = torch.stack([torch.arange(max(s), device=dev) + 0.25 * a for a in range(3)])
    turn = torch.where(torch.arange(max(s), device=dev) < torch.tensor(s, device=dev)[:, None], turn, torch.inf)
    return torch.argsort(turn.flatten())[i] // max(s)


def _rope(st):
    c, pos = st["case"], st["pos"]
    D, half = c["d"], c["d"] // 2
    axis = _axis_of(c, pos.device)
    freq = torch.pow(torch.tensor(c["base"], dtype=torch.float64, device=pos.device),
                     -2.0 * torch.arange(half, dtype=torch.float64, device=pos.device) / D)
    angle = pos.double()[axis].T * freq
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if c["inverse"]:
        sin = -sin
    q, k = st["q"].float(), st["k"].float()
    q = torch.cat([q[..., :half] * cos - q[..., half:] * sin, q[..., half:] * cos + q[..., :half] * sin], -1)
    k = torch.cat([k[..., :half] * cos - k[..., half:] * sin, k[..., half:] * cos + k[..., :half] * sin], -1)
    return q.bfloat16(), k.bfloat16()


def run(st):
    c, op = st["case"], st["case"]["op"]
    if not own:
        plain = {"logp": _logp, "logp_bwd": _logp_bwd, "policy": _policy, "positions": _positions, "rope": _rope}
        return plain[op](st)
    from paper_2602_24082_b200 import binding as B
    plan = st["plan"]
    if op == "logp":
        logp, stats = B.pp_token_logp(plan, st["logits"], st["ids"], temperature=c["temperature"])
        return {"logp": logp, "stats": stats}
    if op == "logp_bwd":
        return B.pp_token_logp_bwd(plan, st["logits"], st["ids"], st["logp"], st["stats"], st["grad"],
                                   temperature=c["temperature"])
    if op == "policy":
        loss, kl, clipped, adv, grad = B.pp_policy_loss(
            plan, st["logp"], st["old"], st["ref"], st["reward"], advantage=c["advantage"], token_mask=st["mask"],
            clip_low=0.2, clip_high=0.28, kl_coef=0.04, reduction=c["reduction"], scale=st["scale"])
        out = {"loss": loss, "kl": kl, "clipped": clipped, "grad": grad}
        return out if adv is None else dict(out, advantage=adv)
    if op == "positions":
        return B.pp_position_ids_axes(plan, st["starts"], st["grids"])[0]
    q, k = st["q"], st["k"]
    if c["inverse"]:
        d_qkv = torch.empty(st["T"], c["hq"] + 2 * c["hkv"], c["d"], dtype=q.dtype, device=q.device)
        q_out, k_out = d_qkv[:, :c["hq"]], d_qkv[:, c["hq"]:c["hq"] + c["hkv"]]
    else:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    return B.pp_rope_qk_axes(plan, q, k, st["pos"], st["sections"], rope_base=c["base"], interleaved=c["interleaved"],
                             inverse=c["inverse"], q_out=q_out, k_out=k_out)


def work(case):
    """Bytes and operations one pass cannot do without: rows of logits that predict something are read,
    all of the gradient's are written."""
    groups = _groups(case)
    T, N, op = _tokens(groups), sum(len(rs) for _, rs in groups), case["op"]
    if op in ("logp", "logp_bwd"):
        _, row = _predicted(groups)
        used, V = len(np.unique(row)), case["vocab"]
        size = 4 if case["type"] == "fp32" else 2
        if op == "logp":
            return {"bytes": used * V * size + 8 * T + 12 * T, "flops": 4 * used * V}
        return {"bytes": used * V * size + T * V * size + 8 * T + 16 * T, "flops": 4 * used * V}
    if op == "policy":
        arrays = 2 + case["old"] + case["ref"]       # log-probabilities in, gradient out
        return {"bytes": 4 * T * arrays + (T if case["masked"] else 0) + (4 * T if case["advantage"] == "token" else 8 * N) + 12 * N,
                "flops": 30 * T}
    if op == "positions":
        return {"bytes": 12 * T + 16 * len(_spans(case, groups)[0]), "flops": 0}
    H, D = case["hq"] + case["hkv"], case["d"]
    return {"bytes": 2 * 2 * T * H * D + 12 * T, "flops": 3 * T * H * D}


# ---------------------------------------------------------------------------- from the definitions, in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    groups = _groups(case)
    T, op, dev = st["T"], case["op"], torch.device("cuda:0")
    temp = case.get("temperature", 1.0)
    if op in ("logp", "logp_bwd"):
        logits, ids = st["logits"], st["ids"].cpu().numpy()
        readers = {}                       # row -> tokens that it predicts
        prompt_last = None
        for a, n, _, k in _segments(groups):
            if k == 0:
                prompt_last = a + n - 1
                continue
            for t in range(a, a + n):
                if ids[t] >= 0:
                    readers.setdefault(prompt_last if t == a else t - 1, []).append(t)
        rows = np.asarray(sorted(readers))
        if op == "logp":
            logp = torch.zeros(T, dtype=torch.float64, device=dev)
            stats = torch.zeros(T, 2, dtype=torch.float64, device=dev)
        else:
            d = torch.zeros(T, case["vocab"], dtype=torch.float64, device=dev)
            grad = st["grad"].double()
        for lo in range(0, len(rows), 512):
            some = rows[lo:lo + 512]
            at = torch.from_numpy(some).to(dev)
            x = logits[at].double() / temp
            lse = torch.logsumexp(x, 1)
            pairs = [(i, t) for i, r in enumerate(some) for t in readers[r]]
            i = torch.tensor([p[0] for p in pairs], device=dev)
            t = torch.tensor([p[1] for p in pairs], device=dev)
            y = st["ids"][t]
            if op == "logp":
                top = x.max(1).values
                stats[at, 0], stats[at, 1] = top, lse - top
                logp[t] = x[i, y] - lse[i]
            else:
                # one reader at a time: (one-hot - softmax) weighted by the reader's gradient
                weight = torch.zeros(len(some), dtype=torch.float64, device=dev)
                weight.scatter_add_(0, i, grad[t])
                part = torch.softmax(x, 1).mul_(-weight[:, None])
                part.view(-1).scatter_add_(0, i * case["vocab"] + y, grad[t])
                d[at] = part / temp
        if op == "logp":
            return {"logp": logp, "stats": stats}
        return d
    if op == "policy":
        get = lambda name: None if st[name] is None else st[name].double().cpu().numpy()
        lp, old, ref, reward = get("logp"), get("old"), get("ref"), get("reward")
        mask = np.ones(T, bool) if st["mask"] is None else st["mask"].cpu().numpy()
        out = {"loss": [], "kl": [], "clipped": [], "advantage": [], "grad": np.zeros(T)}
        a, k = 0, 0
        for p, rs in groups:
            a += p
            r = reward[k:k + len(rs)]
            adv = r
            if case["advantage"] in ("centered", "normalized"):
                adv = r - r.mean()
            if case["advantage"] == "normalized":
                adv = adv / ((r.std(ddof=1) if len(r) > 1 else 0.0) + 1e-6)
            for j, n in enumerate(rs):
                use = np.flatnonzero(mask[a:a + n]) + a
                A = reward[use] if case["advantage"] == "token" else np.full(len(use), adv[j])
                ratio = np.exp(lp[use] - old[use]) if old is not None else np.ones(len(use))
                bound = np.minimum(np.maximum(ratio, 1 - 0.2), 1 + 0.28)
                cut = bound * A < ratio * A
                term, slope = -np.where(cut, bound * A, ratio * A), -np.where(cut, 0, ratio * A)
                kl = np.zeros(len(use))
                if ref is not None:
                    x = ref[use] - lp[use]
                    kl = np.expm1(x) - x
                    term, slope = term + 0.04 * kl, slope + 0.04 * -np.expm1(x)
                w = st["scale"] / (max(1, len(use)) if case["reduction"] == "response" else 1)
                out["loss"].append(w * term.sum())
                out["kl"].append(kl.sum() / max(1, len(use)))
                out["clipped"].append(cut.sum() / max(1, len(use)))
                out["grad"][use] = w * slope
                a += n
            if case["advantage"] != "token":
                out["advantage"] += list(adv)
            k += len(rs)
        if case["advantage"] == "token":
            del out["advantage"]
        return {name: np.asarray(x, np.float64) for name, x in out.items()}
    # positions, counted token by token
    spans = dict(zip(st["starts"].tolist(), st["grids"].tolist()))
    pos = np.zeros((3, T), np.int32)
    after_prompt = 0
    for a, n, _, k in _segments(groups):
        number = after_prompt if k else 0
        t = a
        while t < a + n:
            if t in spans:
                f, h, w = spans[t]
                pos[:, t:t + f * h * w] = number + np.indices((f, h, w)).reshape(3, -1)
                number += max(f, h, w)
                t += f * h * w
            else:
                pos[:, t] = number
                number += 1
                t += 1
        if k == 0:
            after_prompt = number
    if op == "positions":
        return pos
    D, half, s = case["d"], case["d"] // 2, list(st["sections"])
    left, axis = list(s), []
    while len(axis) < half:
        for x in range(3):
            if left[x]:
                take = 1 if case["interleaved"] else left[x]
                axis += [x] * take
                left[x] -= take
    angle = torch.from_numpy(np.stack([pos[axis[i]] * case["base"] ** (-2.0 * i / D) for i in range(half)], 1)).to(dev)
    turn = torch.polar(torch.ones_like(angle), -angle if case["inverse"] else angle)[:, None]
    out = []
    for x in (st["q"], st["k"]):
        y = torch.empty(x.shape, dtype=torch.float64, device=dev)
        for h in range(0, x.shape[1], 8):
            z = torch.complex(x[:, h:h + 8, :half].double(), x[:, h:h + 8, half:].double()) * turn
            y[:, h:h + 8, :half], y[:, h:h + 8, half:] = z.real, z.imag
        out.append(y)
    return tuple(out)
