"""TEST INFRASTRUCTURE: plain numpy fp64 oracle of token log-probabilities and of the clipped policy loss.

Packed rows are split back into the sequences (x, y^k) they stand for (paper Sec. 3.2), so a response's
first token is predicted by the logits of the prompt's last token.  Everything is written out token by
token from the definitions; gradients are the analytic ones.

Pinned by tests/test_oracle_policy_pins.py: torch log_softmax and autograd on unpacked sequences, closed
forms, finite differences.  Shares no code with the CUDA library.
"""
from __future__ import annotations

import numpy as np


def sequences(rows):
    """Per group (prompt tokens, [response tokens, ...]) as ranges of packed indices."""
    t, out = 0, []
    for row in rows:
        for p, rs in row:
            prompt, resp = range(t, t + p), []
            t += p
            for r in rs:
                resp.append(range(t, t + r))
                t += r
            out.append((prompt, resp))
    return out


def predictions(rows):
    """(row of the logits, token it predicts), in the order of the tokens."""
    out = []
    for prompt, resp in sequences(rows):
        for y in resp:
            before = prompt[-1]
            for t in y:
                out.append((before, t))
                before = t
    return out


def token_logp(rows, logits, ids, temperature=1.0):
    """(token_logp [T], row_stats [T, 2]) in fp64."""
    x = np.asarray(logits, np.float64) / temperature
    T, V = x.shape
    logp, stats = np.zeros(T), np.zeros((T, 2))
    with np.errstate(invalid="ignore", over="ignore"):
        for r, t in predictions(rows):
            y = int(ids[t])
            if y < 0:
                continue
            m = x[r].max()
            l = np.log(np.exp(x[r] - m).sum())
            stats[r] = m, l
            logp[t] = x[r, y] - m - l if y < V else np.nan
    return logp, stats


def token_logp_bwd(rows, logits, ids, d_token_logp, temperature=1.0):
    """d_logits [T, V] in fp64, and per element the sum of the magnitudes that were added up."""
    x = np.asarray(logits, np.float64) / temperature
    T, V = x.shape
    d, size = np.zeros((T, V)), np.zeros((T, V))
    for r, t in predictions(rows):
        y = int(ids[t])
        g = float(d_token_logp[t])
        if y < 0 or g == 0.0:
            continue
        p = np.exp(x[r] - x[r].max())
        p /= p.sum()
        part = -g * p
        d[r] += part / temperature
        size[r] += np.abs(part) / temperature
        if y < V:
            # 1 - p of the token itself as the sum of all others
            d[r, y] += g * p[y] / temperature + g * (np.delete(p, y).sum()) / temperature
            size[r, y] += abs(g) * (1 - p[y]) / temperature
    return d, size


def advantages(rows, reward, mode, eps=1e-6):
    r, k, out = np.asarray(reward, np.float64), 0, []
    for _, resp in sequences(rows):
        a = r[k:k + len(resp)].copy()
        if mode != "given":
            a -= a.mean()
        if mode == "normalized":
            a = a / (np.sqrt((a * a).sum() / (len(a) - 1)) + eps) if len(a) > 1 else np.zeros(1)
        out += list(a)
        k += len(resp)
    return np.asarray(out)


def policy_loss(rows, logp, old, ref, reward, mode="normalized", mask=None, clip_low=0.2, clip_high=0.2,
                kl_coef=0.0, reduction="response", scale=1.0, eps=1e-6):
    """(resp_loss, resp_kl, resp_clipped, advantage or None, d_token_logp) in fp64."""
    f = lambda x: None if x is None else np.asarray(x, np.float64)
    lp, old, ref = f(logp), f(old), f(ref)
    adv = None if mode == "token" else advantages(rows, reward, mode, eps)
    T = len(lp)
    loss, kls, cuts, grad = [], [], [], np.zeros(T)
    k = 0
    for _, resp in sequences(rows):
        for y in resp:
            use = [t for t in y if mask is None or mask[t]]
            n = len(use)
            w = scale if reduction == "token" else scale / n if n else 0.0
            total = kl_sum = cut_sum = 0.0
            for t in use:
                A = float(reward[t]) if mode == "token" else adv[k]
                rho = 1.0 if old is None else np.exp(lp[t] - old[t])
                u, v = rho * A, min(max(rho, 1 - clip_low), 1 + clip_high) * A
                term, slope = -min(u, v), 0.0 if v < u else -u
                cut_sum += v < u
                if ref is not None:
                    d = ref[t] - lp[t]
                    # exp(d) - d - 1 as its series where the terms cancel
                    kl = d * d * (0.5 + d * (1 / 6 + d * (1 / 24 + d / 120))) if abs(d) < 1e-3 else np.exp(d) - d - 1
                    kl_sum += kl
                    term += kl_coef * kl
                    slope += kl_coef * -np.expm1(d)
                total += term
                grad[t] = w * slope
            loss.append(w * total)
            kls.append(kl_sum / n if n else 0.0)
            cuts.append(cut_sum / n if n else 0.0)
            k += 1
    return np.asarray(loss), np.asarray(kls), np.asarray(cuts), adv, grad
