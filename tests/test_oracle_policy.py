"""Pins of the oracle of oracle/policy.py: library routines, autograd and
central differences in float64 (CPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import policy as oracle


def test_logits_match_torch_and_its_gradient():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((7, 33)) * 3
    x[2, 5:9] = -np.inf
    y = rng.integers(9, 33, 7).astype(np.int32)
    mask = np.array([1, 1, 1, 0, 1, 1, 1], np.uint8)
    y[5] = -1
    live = [0, 1, 2, 4, 6]
    z = torch.tensor(x * 0.7, requires_grad=True)
    lp = torch.log_softmax(z, 1)
    ent = torch.special.entr(lp.exp()).sum(1)
    got = oracle.logits_logp(x, y, mask, 0.7)
    for r in range(7):
        want = (lp[r, y[r]], ent[r], torch.logsumexp(z[r], 0)) if r in live else (0, 0, 0)
        assert np.allclose(got[:, r], [float(v) for v in (torch.stack(want).detach() if r in live else want)], rtol=1e-13)
    a, c = rng.standard_normal(7), rng.standard_normal(7)
    g = oracle.logits_logp_bwd(x, y, got[2], got[1], a, c, mask, 0.7)
    h = 1e-5
    for r, v in ((0, 3), (0, int(y[0])), (2, 12), (4, 1), (6, int(y[6]))):
        up, down = x.copy(), x.copy()
        up[r, v] += h
        down[r, v] -= h
        f = lambda t: (lambda o: a[r] * o[0, r] + c[r] * o[1, r])(oracle.logits_logp(t, y, mask, 0.7))  # noqa: E731
        assert abs((f(up) - f(down)) / (2 * h) - g[r, v]) < 1e-8
    assert not g[3].any() and not g[5].any() and not g[2, 5:9].any()


def test_logits_gradient_of_a_row_of_lowest_values():
    """Uniform, however little of it an fp32 lse still holds."""
    x = np.full((1, 8), np.finfo(np.float32).min)
    logp, ent, lse = oracle.logits_logp(x, [3])
    assert np.isclose(logp[0], -np.log(8)) and np.isclose(ent[0], np.log(8))
    g = oracle.logits_logp_bwd(x, [3], lse.astype(np.float32), ent, [2.0])
    assert np.allclose(g[0], 2.0 * (np.eye(8)[3] - 1 / 8))


@pytest.mark.parametrize("ratio", ["token", "sequence"])
@pytest.mark.parametrize("reduce", ["tokens", "responses", "sum"])
def test_policy_loss_against_differences(ratio, reduce):
    rng = np.random.default_rng(1)
    B, L = 5, 6
    old, ref = rng.standard_normal((B, L)) * 0.3, rng.standard_normal((B, L)) * 0.3
    lp = old + 0.25 * rng.standard_normal((B, L))
    mask = (rng.random((B, L)) < 0.7).astype(np.uint8)
    mask[3] = 0
    adv = rng.standard_normal(B) if ratio == "sequence" else rng.standard_normal((B, L))
    for kl in ("k1", "k2", "k3"):
        for dual in (0.0, 1.5):
            kw = dict(ratio=ratio, reduce=reduce, kl=kl, clip_low=0.1 if ratio == "token" else 0.03, clip_high=0.15 if ratio == "token" else 0.02, clip_dual=dual, kl_coef=0.3,
                      loss_scale=0.7)
            stats, g, _ = oracle.policy_loss(lp, old, ref, adv, mask, **kw)
            assert stats[4] == mask.sum() and 0 < stats[5] < stats[4]
            h = 1e-6
            for b in range(B):
                for i in range(L):
                    up, down = lp.copy(), lp.copy()
                    up[b, i] += h
                    down[b, i] -= h
                    fd = (oracle.policy_loss(up, old, ref, adv, mask, **kw)[0][0] -
                          oracle.policy_loss(down, old, ref, adv, mask, **kw)[0][0]) / (2 * h)
                    assert abs(fd - g[b, i]) < 1e-7


def test_policy_loss_closed_forms():
    # on-policy without a clip in reach: the plain policy gradient
    adv, mask = np.array([2.0, -1.0]), np.array([[1, 1, 0], [1, 0, 0]])
    lp = -np.ones((2, 3))
    s, g, _ = oracle.policy_loss(lp, None, None, adv, mask, reduce="responses", loss_scale=0.5)
    assert np.allclose(s[:6], [-0.5 * (2.0 - 1.0), -0.5, 0, 0, 3, 0])
    assert np.allclose(g, [[-0.5, -0.5, 0], [0.5, 0, 0]])
    # a gain is held at 1 + clip_high, a loss at 1 - clip_low, a large loss at the second clip
    for d, A, dual, want, cut in ((math.log(2), 1.0, 0, -1.2, 1), (math.log(2), -1.0, 0, 2.0, 0),
                                  (math.log(0.5), -1.0, 0, 0.8, 1), (math.log(0.5), 1.0, 0, -0.5, 0),
                                  (math.log(4), -1.0, 3.0, 3.0, 1)):
        s, g, _ = oracle.policy_loss(np.array([[d]]), np.zeros((1, 1)), None, np.array([A]), np.ones((1, 1)), clip_dual=dual)
        assert np.isclose(s[0], want) and s[5] == cut and (g[0, 0] == 0) == bool(cut)


@pytest.mark.parametrize("kind", ["sigmoid", "hinge", "squared"])
@pytest.mark.parametrize("mean", [False, True])
def test_preference_loss_against_differences(kind, mean):
    rng = np.random.default_rng(2)
    P, L = 6, 4
    w, lo, wr, lr = (rng.standard_normal((P, L)) for _ in range(4))
    wm, lm = ((rng.random((P, L)) < 0.7).astype(np.uint8) for _ in range(2))
    wm[1] = 0
    kw = dict(kind=kind, mean=mean, beta=0.6, margin=0.1, loss_scale=0.3, label_smoothing=0.2 if kind == "sigmoid" else 0)
    o = oracle.preference_loss(w, lo, wr, lr, wm, lm, **kw)
    h = 1e-6
    for arr, name in ((w, "dwin"), (lo, "dlose")):
        for p in range(P):
            for i in range(L):
                v = arr[p, i]
                arr[p, i] = v + h
                up = oracle.preference_loss(w, lo, wr, lr, wm, lm, **kw)["stats"][0]
                arr[p, i] = v - h
                down = oracle.preference_loss(w, lo, wr, lr, wm, lm, **kw)["stats"][0]
                arr[p, i] = v
                assert abs((up - down) / (2 * h) - o[name][p, i]) < 1e-7
    n = np.maximum(wm.sum(1), 1) if mean else np.ones(P)
    assert np.allclose(-o["adv_win"] / n * wm.any(1), np.where(wm.any(1), np.abs(o["dwin"]).max(1) * np.sign(o["dwin"].sum(1)), 0))
    assert np.allclose(o["adv_lose"], -o["adv_win"])


def test_preference_loss_is_dpo():
    """log sigmoid of the scaled difference of log ratios."""
    o = oracle.preference_loss(np.array([[-1.0, -2.0]]), np.array([[-3.0, -1.5]]), np.array([[-1.2, -2.5]]),
                               np.array([[-2.0, -1.0]]), beta=0.5)
    m = 0.5 * ((-3.0 + 3.7) - (-4.5 + 3.0))
    assert np.isclose(o["margins"][0], m) and np.isclose(o["stats"][0], math.log(1 + math.exp(-m)))
