"""Policy and preference losses vs the float64 oracle.

Both sides compute in float64; what differs is the order of sums and the last
places of exp, expm1 and log1p (a few 2^-52 of their values).  With n terms summed,
sums agree within (n + 64) 2^-52 of the sum of the terms' magnitudes, and a ratio or
a margin that hangs on a sum carries that error on.  fp32 outputs add half a step,
2^-24 of the value.
"""
import itertools
import math

import numpy as np
import pytest
import torch

from oracle import policy as oracle

pytestmark = pytest.mark.gpu
E52 = 2.0 ** -52
RATIO, REDUCE, KL = ("token", "sequence"), ("tokens", "responses", "sum"), ("k1", "k2", "k3")
KIND = ("sigmoid", "hinge", "squared")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def lib():
    from paper_2510_11683_amd import bgpo
    return bgpo


def _in(a, pad, dtype=None, offset=0, fill=math.nan):
    """A matrix on the GPU inside a larger one with other values around it."""
    t = torch.from_numpy(np.ascontiguousarray(a))
    t = t if dtype is None else t.to(dtype)
    n, c = t.shape
    big = torch.full((n * (c + pad) + offset,), fill if t.is_floating_point() else 1, dtype=t.dtype, device="cuda")
    v = big[offset:].view(n, c + pad)[:, :c]
    v.copy_(t)
    return v


def _policy_inputs(B, L, dtype, seed=0, per_token=False, empty=True):
    rng = np.random.default_rng([seed, B, L])
    np_t = np.float64 if dtype == torch.float64 else np.float32
    old = (-2.0 * rng.random((B, L))).astype(np_t)
    lp = (old + 0.25 * rng.standard_normal((B, L))).astype(np_t)
    ref = (lp + 0.3 * rng.standard_normal((B, L))).astype(np_t)
    mask = (rng.random((B, L)) < 0.7).astype(np.uint8) * 3       # nonzero counts, whatever the value
    if empty and B > 2:
        mask[B // 2] = 0
    adv = rng.standard_normal((B, L) if per_token else B).astype(np.float32)
    for a in (lp, old, ref) + ((adv,) if per_token else ()):
        a[mask == 0] = np.nan                                    # never read
    return lp, old, ref, adv, mask


def _run_policy(lp, old, ref, adv, mask, dtype, pad=0, grad=True, flags=None, **kw):
    b = lib()
    B, L = lp.shape
    names = dict(ratio=RATIO, reduce=REDUCE, kl=KL)
    prob = b.PolicyLoss(B, L, **{k: names[k].index(v) if k in names else v for k, v in kw.items()})
    big = torch.full((B, L + pad), 77.0, dtype=dtype, device="cuda")
    d = big[:, :L] if grad else None
    stats = torch.full((6,), 5.0, dtype=torch.float64, device="cuda")
    a = _in(adv, pad + 1) if adv.ndim == 2 else torch.from_numpy(adv).cuda()
    b.bgpo_policy_loss(prob, _in(lp, pad, offset=1), None if old is None else _in(old, 2 * pad),
                       None if ref is None else _in(ref, 0), a, _in(mask, 3 * pad, offset=pad), d, stats,
                       b.policy_workspace(prob), flags)
    assert (big[:, L:] == 77.0).all()
    return stats.cpu().numpy(), None if d is None else d.cpu().numpy().astype(np.float64)


def _check_policy(lp, old, ref, adv, mask, dtype, pad=0, **kw):
    want, gw, size = oracle.policy_loss(lp, old, ref, adv, mask, **kw)
    got, g = _run_policy(lp, old, ref, adv, mask, dtype, pad, **kw)
    n = int((mask != 0).sum(1).max()) if kw.get("ratio") == "sequence" else 0
    # (the exponent of a sequence ratio: a mean of n differences of about 1 at most)
    rel = (64 + 2 * n) * E52
    tol = (mask.size + 64) * E52 * size + rel * size
    assert np.abs(got[:4] - want[:4]).max() <= tol + 1e-300, (got, want, tol)
    assert (got[4:] == want[4:]).all()
    # a gradient is the difference of its two terms, each below its own size
    w = kw.get("loss_scale", 1.0)
    terms = np.abs(gw) + abs(w) * abs(kw.get("kl_coef", 0.0)) * 4
    step = 2.0 ** -24 if dtype == torch.float32 else 0.0
    err = np.abs(g - gw)
    assert (err <= step * np.abs(gw) + rel * terms + 2.0 ** -150).all(), (err - step * np.abs(gw)).max()
    assert (g[mask == 0] == 0).all()
    return got


SIZES = [(1, 1), (1, 7), (3, 1), (8, 64), (8, 512), (5, 1000), (2, 5003), (1, 70001), (300, 33), (5000, 3), (2500, 65),
         (40, 1025), (4, 16385), (3, 33000)]


@pytest.mark.parametrize("B,L", SIZES)
def test_policy_loss(B, L):
    combos = list(itertools.product(RATIO, REDUCE, KL, (torch.float32, torch.float64)))
    rng = np.random.default_rng([B, L])
    for k in rng.permutation(len(combos))[:6 if B * L < 50000 else 3]:
        ratio, reduce, kl, dtype = combos[k]
        lp, old, ref, adv, mask = _policy_inputs(B, L, dtype, seed=int(k), per_token=ratio == "token" and bool(k % 2))
        _check_policy(lp, old, ref, adv, mask, dtype, pad=int(k % 4), ratio=ratio, reduce=reduce, kl=kl, clip_low=0.1,
                      clip_high=0.25, clip_dual=3.0 if k % 3 else 0.0, kl_coef=0.05, loss_scale=1.0 / B)


@pytest.mark.parametrize("ratio", RATIO)
@pytest.mark.parametrize("reduce", REDUCE)
def test_policy_loss_options(ratio, reduce):
    """Every combination at one ragged size; without old, reference, gradient."""
    B, L = 21, 70
    for kl, dtype in itertools.product(KL, (torch.float32, torch.float64)):
        lp, old, ref, adv, mask = _policy_inputs(B, L, dtype, seed=3)
        kw = dict(ratio=ratio, reduce=reduce, kl=kl, clip_low=0.02 if ratio == "sequence" else 0.2,
                  clip_high=0.01 if ratio == "sequence" else 0.1, loss_scale=0.125)
        got = _check_policy(lp, old, ref, adv, mask, dtype, kl_coef=0.1, **kw)
        assert 0 < got[5] < got[4]
        _check_policy(lp, old, None, adv, mask, dtype, **kw)
        on = _check_policy(lp, None, ref, adv, mask, dtype, **kw)      # on-policy: nothing is cut, d = 0
        assert on[5] == 0 and on[3] == 0
        alone, none = _run_policy(lp, old, ref, adv, mask, dtype, grad=False, kl_coef=0.1, **kw)
        assert none is None and np.array_equal(alone, got)
        _check_policy(lp, old, ref, adv, mask, dtype, **{**kw, "clip_high": math.inf, "clip_low": 1.0})


def test_policy_loss_without_positions():
    for ratio, reduce in itertools.product(RATIO, REDUCE):
        lp, old, ref, adv, _ = _policy_inputs(9, 40, torch.float32)
        mask = np.zeros((9, 40), np.uint8)
        flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        s, g = _run_policy(lp * np.nan, old, ref, adv, mask, torch.float32, flags=flags, ratio=ratio, reduce=reduce, kl_coef=1.0)
        assert not s.any() and not g.any() and int(flags) == 0


def test_policy_loss_border_values():
    """Ratios at the borders and one float64 step past them: a tie keeps its gradient."""
    edge = [math.log(1.25), math.log(0.75)]
    ds = [v for e in edge for v in (e, np.nextafter(e, 9), np.nextafter(e, -9))] + [0.0]
    lp = np.array([ds, ds])
    old, adv, mask = np.zeros_like(lp), np.array([1.0, -1.0], np.float32), np.ones(lp.shape, np.uint8)
    s, g = _run_policy(lp, old, None, adv, mask, torch.float64, reduce="sum", clip_low=0.25, clip_high=0.25)
    r = torch.exp(torch.from_numpy(lp).cuda()).cpu().numpy()      # the same exponential
    want = np.stack((np.where(r[0] > 1.25, 0, -r[0]), np.where(r[1] < 0.75, 0, r[1])))
    assert np.allclose(g, want, rtol=4 * E52, atol=0) and s[5] == (want == 0).sum()


def test_policy_loss_flags_what_is_not_finite():
    b = lib()
    lp, old, ref, adv, mask = _policy_inputs(4, 50, torch.float32, empty=False)
    mask[:] = 1
    lp, old, ref = (np.nan_to_num(v) for v in (lp, old, ref))
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    adv[:] = [1.0, -1.0, 1.0, -1.0]
    _run_policy(lp, old, ref, adv, mask, torch.float32, flags=flags)
    assert int(flags) == 0
    far = lp.copy()
    far[0, 3] = 800.0                                       # a gain past every float: clipped, finite
    s, g = _run_policy(far, old, None, adv, mask, torch.float32, flags=flags)
    assert np.isfinite(s).all() and g[0, 3] == 0 and int(flags) == 0
    far[1, 3] = 800.0                                       # a loss past every float is none
    s, _ = _run_policy(far, old, None, adv, mask, torch.float32, flags=flags)
    assert s[0] == math.inf and int(flags) == b.BGPO_FLAG_NONFINITE
    flags.zero_()
    lp[2, 2] = np.nan
    s, g = _run_policy(lp, old, ref, adv, mask, torch.float32, flags=flags)
    assert math.isnan(s[0]) and np.isnan(g).sum() == 1 and int(flags) == b.BGPO_FLAG_NONFINITE
    flags.zero_()                                           # finite terms, an fp32 gradient past its range
    s, g = _run_policy(old + np.float32(80), old, None, -adv ** 2, mask, torch.float32, flags=flags, reduce="sum", loss_scale=1e10)
    assert np.isfinite(s).all() and np.isinf(g).all() and int(flags) == b.BGPO_FLAG_NONFINITE


@pytest.mark.parametrize("L", [3, 70, 700])
def test_infinite_objective_of_a_sequence_ratio(L):
    """A ratio past every float under a negative advantage: the loss is +inf, not NaN,
    also where lanes of the response's group have no position."""
    b = lib()
    old = np.zeros((2, L))
    lp = old.copy()
    lp[1] = 900.0
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    s, g = _run_policy(lp, old, None, np.array([1.0, -2.0], np.float32), np.ones((2, L), np.uint8), torch.float64, flags=flags,
                       ratio="sequence", reduce="responses")
    assert s[0] == math.inf and s[1] == math.inf and int(flags) == b.BGPO_FLAG_NONFINITE
    assert np.isfinite(g[0]).all() and (g[1] == math.inf).all()


# ---------------------------------------------------------------- preference loss

def _run_pref(a, dtype, pad=0, grad=True, adv=True, margins=True, flags=None, **kw):
    b = lib()
    P, L = a["win"].shape
    prob = b.PreferenceLoss(P, L, **{k: KIND.index(v) if k == "kind" else v for k, v in kw.items()})
    t = {k: None if v is None else _in(v, pad * (i % 3), offset=i % 2) for i, (k, v) in enumerate(a.items())}
    big = torch.full((2, P, L + pad), 77.0, dtype=dtype, device="cuda")
    d = [v[:, :L] for v in big] if grad else [None, None]
    av = [torch.full((P,), 9.0, device="cuda") for _ in range(2)] if adv else [None, None]
    m = torch.full((P,), 9.0, dtype=torch.float64, device="cuda") if margins else None
    stats = torch.full((3,), 9.0, dtype=torch.float64, device="cuda")
    b.bgpo_preference_loss(prob, t["win"], t["lose"], t["win_ref"], t["lose_ref"], t["win_mask"], t["lose_mask"], d[0], d[1],
                           m, av[0], av[1], stats, b.preference_workspace(prob), flags)
    assert (big[:, :, L:] == 77.0).all()
    return {k: None if v is None else v.cpu().numpy().astype(np.float64)
            for k, v in dict(stats=stats, margins=m, adv_win=av[0], adv_lose=av[1], dwin=d[0], dlose=d[1]).items()}


def _pref_inputs(P, L, dtype, ref, masks, seed=0):
    rng = np.random.default_rng([seed, P, L])
    np_t = np.float64 if dtype == torch.float64 else np.float32
    a = {k: (-2 * rng.random((P, L)) + rng.standard_normal((P, 1)) / math.sqrt(L)).astype(np_t) for k in ("win", "lose")}
    a.update({k + "_ref": (a[k] + 0.3 * rng.standard_normal((P, L))).astype(np_t) if ref else None for k in ("win", "lose")})
    a.update({k + "_mask": (rng.random((P, L)) < 0.6).astype(np.uint8) * 2 if masks else None for k in ("win", "lose")})
    if masks:
        if P > 1:
            a["win_mask"][P // 2] = 0
            a["lose_mask"][P - 1] = 0
        for k in ("win", "lose"):
            for v in (a[k], a[k + "_ref"]):
                if v is not None:
                    v[a[k + "_mask"] == 0] = np.nan
    return a


def _check_pref(a, dtype, pad=0, **kw):
    want = oracle.preference_loss(**{k: None if v is None else v for k, v in a.items()}, **kw)
    got = _run_pref(a, dtype, pad, **kw)
    L = a["win"].shape[1]
    m, beta, scale = want["margins"], kw.get("beta", 0.1), abs(kw.get("loss_scale", 1.0))
    tm = (L + 64) * E52 * (want["size"] + np.abs(m) + abs(kw.get("margin", 0.0)))       # the margins' error
    assert (np.abs(got["margins"] - m) <= tm).all()
    # losses and their derivatives change by at most `slope` and `curve` times that
    v = np.abs(m - 0.5) / beta
    slope = 1.0 if kw["kind"] != "squared" else 2 * (v + 1) / beta
    curve = {"sigmoid": 0.25, "hinge": 0.0, "squared": 2 / beta ** 2}[kw["kind"]]
    lt = scale * (slope * tm + 64 * E52 * (1 + np.abs(m) + (v * v if kw["kind"] == "squared" else 0)))
    assert abs(got["stats"][0] - want["stats"][0]) <= lt.sum() + len(m) * E52 * abs(want["stats"][0])
    sure = np.abs(m) > tm                          # (a margin of 0 within its error may count either way)
    assert abs(got["stats"][1] - want["stats"][1]) <= (~sure).sum()
    assert abs(got["stats"][2] - want["stats"][2]) <= tm.sum() + (len(m) + 64) * E52 * np.abs(m).sum()
    gt = scale * beta * (curve * tm + 64 * E52 * slope)
    for k in ("adv_win", "adv_lose"):
        assert (np.abs(got[k] - want[k]) <= gt + 2.0 ** -24 * np.abs(want[k])).all()
    step = 2.0 ** -24 if dtype == torch.float32 else 0.0
    for k in ("dwin", "dlose"):
        gg = np.broadcast_to(gt, m.shape)[:, None]
        assert (np.abs(got[k] - want[k]) <= gg + step * np.abs(want[k])).all()
        if a[k[1:] + "_mask"] is not None:
            assert (got[k][a[k[1:] + "_mask"] == 0] == 0).all()
    return got


@pytest.mark.parametrize("P,L", [(1, 1), (1, 33), (4, 16), (8, 64), (3, 1000), (2, 9001), (1, 70001), (257, 129), (3000, 5), (2100, 70)])
def test_preference_loss(P, L):
    combos = list(itertools.product(KIND, (False, True), (False, True), (False, True), (torch.float32, torch.float64)))
    rng = np.random.default_rng([P, L])
    for k in rng.permutation(len(combos))[:8 if P * L < 50000 else 3]:
        kind, mean, ref, masks, dtype = combos[k]
        _check_pref(_pref_inputs(P, L, dtype, ref, masks, int(k)), dtype, pad=int(k % 3), kind=kind, mean=mean, beta=0.3,
                    margin=0.2 if k % 2 else 0.0, label_smoothing=0.1 if kind == "sigmoid" and k % 3 else 0.0, loss_scale=1.0 / P)


def test_preference_loss_parts_and_interleaved_pairs():
    b = lib()
    P, L = 9, 37
    a = _pref_inputs(P, L, torch.float32, True, False)
    whole = _run_pref(a, torch.float32, kind="sigmoid")
    for off in ("grad", "adv", "margins"):
        part = _run_pref(a, torch.float32, kind="sigmoid", **{off: False})
        assert all(np.array_equal(part[k], whole[k]) for k in whole if part[k] is not None)
    # responses 2p and 2p + 1 of one array, gradients and advantages likewise
    x = torch.empty(2 * P, L, device="cuda")
    r = torch.empty_like(x)
    x[0::2], x[1::2] = torch.from_numpy(a["win"]).cuda(), torch.from_numpy(a["lose"]).cuda()
    r[0::2], r[1::2] = torch.from_numpy(a["win_ref"]).cuda(), torch.from_numpy(a["lose_ref"]).cuda()
    d, adv = torch.empty_like(x), torch.empty(2 * P, device="cuda")
    stats = torch.empty(3, dtype=torch.float64, device="cuda")
    prob = b.PreferenceLoss(P, L)
    b.bgpo_preference_loss(prob, x[0::2], x[1::2], r[0::2], r[1::2], None, None, d[0::2], d[1::2], None, adv[0::2], adv[1::2],
                           stats, b.preference_workspace(prob))
    assert np.array_equal(stats.cpu().numpy(), whole["stats"])
    assert np.array_equal(d[0::2].cpu().numpy(), whole["dwin"]) and np.array_equal(d[1::2].cpu().numpy(), whole["dlose"])
    assert np.array_equal(adv[0::2].cpu().numpy(), whole["adv_win"]) and np.array_equal(adv[1::2].cpu().numpy(), whole["adv_lose"])


def test_preference_loss_at_its_limits():
    """Margins past every exponential, and what is not finite."""
    b = lib()
    a = {k: np.zeros((4, 2), np.float64) for k in ("win", "lose")}
    a.update(win_ref=None, lose_ref=None, win_mask=None, lose_mask=None)
    a["win"][:, 0] = [5000.0, -5000.0, 0.0, 1.0]
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    o = _run_pref(a, torch.float64, flags=flags, kind="sigmoid", beta=1.0)
    assert abs(o["stats"][0] - (5000.0 + math.log(2) + math.log1p(math.exp(-1)))) < 1e-9
    assert o["stats"][1] == 2 and o["adv_win"][1] == 1.0 and abs(o["adv_win"][0]) == 0 and int(flags) == 0
    o = _run_pref(a, torch.float64, flags=flags, kind="hinge", beta=1.0)
    assert o["stats"][0] == 5001.0 + 1.0 and o["adv_win"].tolist() == [0, 1, 1, 0] and int(flags) == 0   # m = 1 exactly: 0
    # an advantage past fp32's range is flagged where it is asked for
    o = _run_pref(a, torch.float64, flags=flags, kind="squared", beta=1e-3, loss_scale=1e36, adv=False)
    assert int(flags) == 0 and np.isfinite(o["dwin"]).all()
    o = _run_pref(a, torch.float64, flags=flags, kind="squared", beta=1e-3, loss_scale=1e36)
    assert int(flags) == b.BGPO_FLAG_NONFINITE and np.isinf(o["adv_win"]).any()
    flags.zero_()
    a["lose"][2, 1] = np.nan
    o = _run_pref(a, torch.float64, flags=flags, kind="hinge", beta=1.0)
    assert math.isnan(o["stats"][0]) and np.isnan(o["dwin"][2]).all() and int(flags) == b.BGPO_FLAG_NONFINITE


# ---------------------------------------------------------------- calls

def test_calls_are_deterministic_and_replay():
    """The same bits from a second call and from replays of a captured graph, with
    eager work between them and a workspace of other values."""
    b = lib()
    for B, L in ((8, 512), (3, 20000), (700, 900)):
        gen = torch.Generator(device="cuda").manual_seed(B)
        old, lp, ref = (torch.empty(B, L, device="cuda") for _ in range(3))
        mask = torch.empty(B, L, dtype=torch.bool, device="cuda")
        adv = torch.randn(B, device="cuda", generator=gen)
        d, dw, dl = (torch.empty(B, L, device="cuda") for _ in range(3))
        stats, ps = (torch.empty(n, dtype=torch.float64, device="cuda") for n in (6, 3))
        margins = torch.empty(B, dtype=torch.float64, device="cuda")
        probs = [b.PolicyLoss(B, L, ratio=k, reduce=r, kl_coef=0.1) for k in (0, 1) for r in (0, 1)]
        pp = b.PreferenceLoss(B, L)
        ws, pws = b.policy_workspace(probs[0]), b.preference_workspace(pp)
        outs = (d, dw, dl, stats, ps, margins)

        def fill():
            for t in (old, lp, ref):
                t.copy_(torch.randn(B, L, device="cuda", generator=gen))
            mask.copy_(torch.rand(B, L, device="cuda", generator=gen) < 0.6)

        for prob in probs:
            def step():
                b.bgpo_policy_loss(prob, lp, old, ref, adv, mask, d, stats, ws)
                b.bgpo_preference_loss(pp, lp, old, ref, ref, mask, mask, dw, dl, margins, None, None, ps, pws)

            fill()
            step()
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
            for _ in range(2):
                fill()
                got = []
                for run in (step, step, g.replay):
                    for t in outs + (ws, pws):
                        t.fill_(99)
                    run()
                    torch.cuda.synchronize()
                    got.append([t.clone() for t in outs])
                assert all(torch.equal(p, q) for o in got[1:] for p, q in zip(got[0], o))


def test_exponentials_over_their_range():
    """The kernels' own e^x and e^x - 1 through the loss's gradient (fp64, one
    position to a weight of 1).  The series leaves 2^-50.8 |f| <= 1.1 2^-52 of e^f, its
    Horner steps and the final sum about 2.5 more: 6 2^-52 of e^x; of e^x - 1 that is up
    to 3.4 times as much where 2^n first differs from 1 (|x| near 0.35)."""
    rng = np.random.default_rng(9)
    x = np.concatenate([np.linspace(-760, 712, 4001), rng.uniform(-1, 1, 3000), 10.0 ** rng.uniform(-18, 0, 2000),
                        -10.0 ** rng.uniform(-18, 0, 2000), [0.0, 709.78, 709.79, -745.1, -745.2, -np.inf, np.inf]])
    for L in (len(x), 512):                                  # the long rows' kernel and the small batch's
        v = x[:L] if L < len(x) else x
        z, one, on = np.zeros((1, len(v))), np.ones(1, np.float32), np.ones((1, len(v)), np.uint8)
        _, g = _run_policy(v[None].copy(), z, None, one, on, torch.float64, reduce="sum", clip_low=1.0, clip_high=math.inf)
        with np.errstate(over="ignore"):
            want = np.exp(v)
        fin = np.isfinite(want)
        assert np.array_equal(-g[0][~fin], want[~fin])
        assert (np.abs(-g[0][fin] - want[fin]) <= 6 * E52 * want[fin] + 2.0 ** -1073).all()
        # q = ref - logp, no policy term: d KL / d logp = -(e^q - 1)
        _, g = _run_policy(z.copy(), None, v[None].copy(), 0 * one, on, torch.float64, reduce="sum", kl="k3", kl_coef=1.0)
        with np.errstate(over="ignore"):
            want = np.expm1(v)
        assert np.array_equal(-g[0][~fin], want[~fin])
        assert (np.abs(-g[0][fin] - want[fin]) <= 20 * E52 * np.abs(want[fin]) + 2.0 ** -1073).all()


@pytest.mark.parametrize("where", ["prompt", "gap", "one", "last"])
def test_long_rows_by_where_they_count(where):
    """Masks whose live range starts late, has a gap, is one position, or ends with
    the row; lengths about every step of the long rows' kernel."""
    for L in (513, 516, 1023, 1024, 1025, 2050, 4099):
        lp, old, ref, adv, mask = _policy_inputs(3, L, torch.float32, seed=7, empty=False)
        lp, old, ref = (np.nan_to_num(v, nan=-1.0) for v in (lp, old, ref))
        mask[:] = 0
        if where == "prompt":
            mask[0, L // 3:], mask[1, L // 2: L - 5], mask[2, 1:] = 1, 1, 1
        elif where == "gap":
            mask[0, :7], mask[0, L - 9:], mask[1, 255:258], mask[2, ::97] = 1, 1, 1, 1
        elif where == "one":
            mask[0, 0], mask[1, L - 1], mask[2, L // 2] = 1, 1, 1
        else:
            mask[0, L - 1], mask[1, L - 4:], mask[2, L - 6: L - 1] = 1, 1, 1
        for a in (lp, old, ref):
            a[mask == 0] = np.nan
        for ratio, reduce in itertools.product(RATIO, REDUCE):
            _check_policy(lp, old, ref, adv, mask, torch.float32, pad=1, ratio=ratio, reduce=reduce, clip_low=0.1, kl_coef=0.1)
        a = dict(win=lp, lose=old, win_ref=ref, lose_ref=ref, win_mask=mask, lose_mask=np.roll(mask, 1, 0))
        for k in ("lose", "lose_ref"):
            a[k] = np.where(a["lose_mask"] == 0, np.float32(np.nan), np.nan_to_num(a[k], nan=-1.5)).astype(np.float32)
        for mean in (False, True):
            _check_pref(a, torch.float32, pad=1, kind="sigmoid", mean=mean)


@pytest.mark.parametrize("L", [40, 700, 4099])
def test_rows_far_apart(L):
    """Responses more than 2^32 bytes apart, and beyond 2^31 elements: the bits of
    the same responses packed."""
    b = lib()
    B, ld = 3, (1 << 30) + 3
    g = torch.Generator(device="cuda").manual_seed(L)
    r = lambda: -torch.randn(B, L, generator=g, device="cuda").abs()  # noqa: E731
    lp, old = r(), r()
    adv = torch.randn(B, generator=g, device="cuda")
    mask = torch.rand(B, L, generator=g, device="cuda") < 0.8
    big, big_out = (torch.empty((B - 1) * ld + L, device="cuda") for _ in range(2))
    far, out = (torch.as_strided(t, (B, L), (ld, 1)) for t in (big, big_out))
    far.copy_(lp)
    prob = b.PolicyLoss(B, L, ratio=b.BGPO_RATIO_SEQUENCE, reduce=b.BGPO_REDUCE_RESPONSES)
    ws = b.policy_workspace(prob)
    res = []
    for x, d in ((lp, torch.empty_like(lp)), (far, out)):
        stats = torch.empty(6, dtype=torch.float64, device="cuda")
        b.bgpo_policy_loss(prob, x, old, None, adv, mask, d, stats, ws)
        res.append((stats.cpu(), d.contiguous().cpu()))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])
    pref = b.PreferenceLoss(B, L)
    ws = b.preference_workspace(pref)
    res = []
    for x, d in ((lp, torch.empty_like(lp)), (far, out)):
        stats = torch.empty(3, dtype=torch.float64, device="cuda")
        dlo = torch.empty_like(old)
        b.bgpo_preference_loss(pref, x, old, None, None, mask, mask, d, dlo, None, None, None, stats, ws)
        res.append((stats.cpu(), d.contiguous().cpu(), dlo.cpu()))
    assert all(torch.equal(p, q) for p, q in zip(*res))
