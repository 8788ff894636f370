"""The oracle of token log-probabilities and of the policy loss against torch on unpacked sequences,
closed forms and finite differences."""
import numpy as np
import pytest
import torch

from oracle import policy as P

ROWS = [[(3, (4, 1, 2))], [(1, (5,)), (6, (1, 1))]]
T = sum(p + sum(rs) for row in ROWS for p, rs in row)
N = sum(len(rs) for row in ROWS for _, rs in row)


def _logits(V=11, seed=0):
    rng = np.random.default_rng(seed)
    return rng.normal(size=(T, V)) * 3, rng.integers(0, V, T)


@pytest.mark.parametrize("temperature", [1.0, 0.7])
def test_token_logp_and_gradient_are_those_of_the_unpacked_sequences(temperature):
    x, ids = _logits()
    g = np.random.default_rng(1).normal(size=T)
    want, leaf = np.zeros(T), torch.tensor(x, requires_grad=True)
    total = 0
    for prompt, resp in P.sequences(ROWS):
        for y in resp:
            seq = torch.tensor(list(prompt) + list(y))      # the sequence (x, y^k), shifted by one
            lp = torch.log_softmax(leaf[seq[:-1]] / temperature, -1)
            lp = lp[torch.arange(len(lp)), torch.tensor(ids)[seq[1:]]][len(prompt) - 1:]
            want[list(y)] = lp.detach().numpy()
            total = total + (lp * torch.tensor(g[list(y)])).sum()
    total.backward()
    got, stats = P.token_logp(ROWS, x, ids, temperature)
    assert np.abs(got - want).max() < 1e-12
    d, size = P.token_logp_bwd(ROWS, x, ids, g, temperature)
    assert np.abs(d - leaf.grad.numpy()).max() < 1e-12
    assert (size >= np.abs(d) - 1e-12).all()
    used = sorted({r for r, _ in P.predictions(ROWS)})
    lse = torch.logsumexp(torch.tensor(x) / temperature, -1).numpy()
    assert np.abs(stats.sum(1)[used] - lse[used]).max() < 1e-12
    assert not np.delete(stats, used, 0).any() and not np.delete(d, used, 0).any()


def test_negative_ids_do_not_count_and_ids_beyond_are_nan():
    x, ids = _logits()
    ids[4], ids[5] = -100, 11
    lp, _ = P.token_logp(ROWS, x, ids)
    assert lp[4] == 0 and np.isnan(lp[5])
    d, _ = P.token_logp_bwd(ROWS, x, ids, np.eye(T)[4])
    assert not d.any()


def test_policy_loss_closed_forms():
    rng = np.random.default_rng(2)
    lp = -rng.exponential(size=T)
    r = rng.normal(size=N)
    # no old policy and no reference: the plain policy gradient with the reward as advantage
    loss, kl, cut, adv, grad = P.policy_loss(ROWS, lp, None, None, r, "given", scale=0.5)
    spans = [list(y) for _, resp in P.sequences(ROWS) for y in resp]
    assert np.allclose(loss, -0.5 * r) and not kl.any() and not cut.any() and np.allclose(adv, r)
    for k, y in enumerate(spans):
        assert np.allclose(grad[y], -0.5 * r[k] / len(y))
    # a group of one has no advantage
    assert P.advantages([[(2, (3,))]], [7.0], "normalized") == 0 and P.advantages([[(2, (3,))]], [7.0], "centered") == 0
    a = P.advantages([[(2, (3, 1, 1))]], [1.0, 2.0, 4.0], "normalized", 0.0)
    assert np.allclose(a, (np.array([1, 2, 4]) - 7 / 3) / np.std([1, 2, 4], ddof=1))


@pytest.mark.parametrize("mode", ["given", "centered", "normalized", "token"])
@pytest.mark.parametrize("reduction", ["response", "token"])
def test_policy_gradient_is_that_of_autograd_and_of_differences(mode, reduction):
    rng = np.random.default_rng(3)
    lp = -rng.exponential(size=T)
    old, ref = lp + 0.3 * rng.normal(size=T), lp + 0.2 * rng.normal(size=T)
    reward = rng.normal(size=T if mode == "token" else N)
    mask = rng.random(T) < 0.8
    mask[ROWS[0][0][0]:ROWS[0][0][0] + 4] = False           # a response with nothing left
    kw = dict(mode=mode, mask=mask, clip_low=0.2, clip_high=0.28, kl_coef=0.04, reduction=reduction, scale=0.3)
    loss, kl, cut, adv, grad = P.policy_loss(ROWS, lp, old, ref, reward, **kw)
    assert loss[0] == kl[0] == cut[0] == 0
    leaf = torch.tensor(lp, requires_grad=True)
    total, k = 0, 0
    for _, resp in P.sequences(ROWS):
        for y in resp:
            use = [t for t in y if mask[t]]
            A = torch.tensor(reward[use]) if mode == "token" else adv[k]
            rho = torch.exp(leaf[use] - torch.tensor(old[use]))
            d = torch.tensor(ref[use]) - leaf[use]
            l = -torch.minimum(rho * A, rho.clamp(0.8, 1.28) * A) + 0.04 * (d.exp() - d - 1)
            if use:
                l = 0.3 * (l.mean() if reduction == "response" else l.sum())
                assert abs(float(l) - loss[k]) < 1e-12
                total = total + l
            k += 1
    total.backward()
    assert np.abs(leaf.grad.numpy() - grad).max() < 1e-12
    h = 1e-6
    for t in rng.permutation(T)[:8]:
        e = h * np.eye(T)[t]
        up, down = (P.policy_loss(ROWS, lp + s * e, old, ref, reward, **kw)[0].sum() for s in (1, -1))
        assert abs((up - down) / (2 * h) - grad[t]) < 1e-6
