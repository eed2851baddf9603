"""The operators together, as an update uses them.

* token log-probabilities of logits -> clipped policy loss -> gradient of the
  logits -> norm -> clipping, against autograd in float64;
* ELBO forwards of two policies (bgpo_elbo_fwd) -> preference loss -> its
  advantages through bgpo_elbo_bwd_accumulate -> norm and clipping of dX and dW,
  against the float64 ELBO oracle; and the clipped ratio of ELBO estimates.
"""
import numpy as np
import pytest
import torch

import workloads
from oracle import elbo
from oracle import policy as oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def lib():
    from paper_2510_11683_amd import bgpo
    return bgpo


def _token_step(b, x, y, old, ref, adv, mask, max_norm, B, L, scale, bufs):
    """One step over logits x [B L, V]; dlogits in place of a copy of them."""
    n = B * L
    V = x.shape[1]
    live = mask.view(-1)
    b.bgpo_logits_logp(x, y, bufs["logp"], bufs["ent"], bufs["lse"], bufs["lws"], row_mask=live, scale=scale)
    prob = b.PolicyLoss(B, L, clip_low=0.05, clip_high=0.05, kl_coef=0.1)
    b.bgpo_policy_loss(prob, bufs["logp"].view(B, L), old, ref, adv, mask, bufs["dlogp"].view(B, L), bufs["stats"], bufs["pws"],
                       bufs["flags"])
    b.bgpo_logits_logp_bwd(x, y, bufs["lse"], bufs["ent"], bufs["dlogp"], bufs["dent"], bufs["dx"], row_mask=live, scale=scale)
    assert bufs["dx"].shape == (n, V)
    b.bgpo_grad_norm(bufs["list"], bufs["norm"], bufs["gws"], status_flags=bufs["flags"])
    b.bgpo_grad_clip(bufs["list"], max_norm, bufs["norm"])


def test_token_update_matches_autograd():
    b = lib()
    B, L, V, scale, c_ent = 6, 37, 1203, 0.8, 0.02
    rng = np.random.default_rng(11)
    x64 = torch.from_numpy(rng.standard_normal((B * L, V)).astype(np.float32)).double()
    yn = rng.integers(0, V, B * L).astype(np.int32)
    mask = (np.arange(L)[None] < rng.integers(1, L + 1, B)[:, None])
    mask[2] = False
    z = x64.clone().requires_grad_(True)
    lp = torch.log_softmax(z * scale, 1)
    ent = torch.special.entr(lp.exp()).sum(1)
    logp = lp.gather(1, torch.from_numpy(yn).long()[:, None])[:, 0].view(B, L)
    old = (logp.detach() + 0.08 * torch.from_numpy(rng.standard_normal((B, L)))).float()
    ref = (logp.detach() + 0.1 * torch.from_numpy(rng.standard_normal((B, L)))).float()
    adv = torch.from_numpy(rng.standard_normal(B).astype(np.float32))
    m = torch.from_numpy(mask)
    r = (logp - old.double()).exp()
    A = adv.double()[:, None]
    obj = torch.minimum(r * A, r.clamp(0.95, 1.05) * A)
    q = ref.double() - logp
    N = m.sum()
    loss = ((-obj + 0.1 * (q.exp() - q - 1)) * m).sum() / N
    total = loss - c_ent * (ent.view(B, L) * m).sum() / N
    (want,) = torch.autograd.grad(total, z)
    norm = float(want.norm())
    max_norm = 0.4 * norm

    x = x64.float().cuda()
    f = lambda n, t=torch.float32: torch.empty(n, dtype=t, device="cuda")  # noqa: E731
    mc = m.cuda()
    bufs = dict(logp=f(B * L), ent=f(B * L), lse=f(B * L), dlogp=f(B * L), stats=f(6, torch.float64), norm=f(1, torch.float64),
                dent=torch.full((B * L,), -c_ent / float(N), device="cuda"), dx=torch.empty_like(x),
                flags=torch.zeros(1, dtype=torch.int32, device="cuda"), lws=b.logits_workspace(B * L, V),
                pws=b.policy_workspace(b.PolicyLoss(B, L)), gws=b.grad_workspace())
    bufs["list"] = b.GradList([bufs["dx"]])
    args = (b, x, torch.from_numpy(yn).cuda(), old.cuda(), ref.cuda(), adv.cuda(), mc, max_norm, B, L, scale, bufs)
    _token_step(*args)
    # fp32 log-probabilities of about 7 (2^-24 of them and of the sums, about 1e-6) make ratios, and with
    # them gradients, off by as much
    assert abs(float(bufs["stats"][0]) - float(loss)) < 1e-5 * (1 + abs(float(loss)))
    assert abs(float(bufs["norm"]) - norm) < 1e-5 * norm and int(bufs["flags"]) == 0
    got = bufs["dx"].double().cpu()
    ref_g = want * (max_norm / norm)
    assert float((got - ref_g).norm()) < 1e-5 * float(ref_g.norm())
    assert (got[~m.view(-1)] == 0).all()
    eager = {k: bufs[k].clone() for k in ("logp", "stats", "norm", "dx")}
    # the whole update as one graph
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _token_step(*args)
    for _ in range(3):
        for k in eager:
            bufs[k].fill_(1.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(bufs[k], v) for k, v in eager.items())


def _elbos(b, prob, dev, W):
    B, nt = prob.B, prob.n_t
    ell = torch.zeros(B, nt, dtype=torch.float64, device="cuda")
    nm = torch.zeros(B, nt, dtype=torch.int32, device="cuda")
    b.bgpo_elbo_fwd(prob, dev["hidden"], W, dev["targets"], dev["resp_mask"], ell, nm, None, b.alloc_workspace(prob))
    return ell


def _old_weights(x):
    """Head weights of the policy before the update: other by a fifth of their size."""
    W = workloads.bf16_bits_to_f32(x["W"])
    return W + 0.004 * np.random.default_rng(3).standard_normal(W.shape).astype(np.float32)


@pytest.mark.parametrize("kind", ["preference", "clipped"])
def test_elbo_update_matches_the_oracle(kind):
    b = lib()
    w = workloads.TINY.replace(B=6, n_t=8)
    x = workloads.generate(w)
    dev = b.device_inputs(x)
    B, L, d, V, nt = w.B, w.L, w.d, w.V, w.n_t
    prob = b.Problem(B, L, d, V, nt, seed=w.philox_seed, seq_id_base=w.seq_id_base, bound=b.BGPO_BOUND_TAYLOR)
    W_old = torch.from_numpy(_old_weights(x)).cuda().bfloat16().view(dev["W"].dtype)
    ell, ref = _elbos(b, prob, dev, dev["W"]), _elbos(b, prob, dev, W_old)
    adv = torch.empty(B, device="cuda")
    if kind == "preference":
        P = B // 2
        pp = b.PreferenceLoss(P, nt, mean=True, beta=0.5, loss_scale=1.0 / P)
        stats = torch.empty(3, dtype=torch.float64, device="cuda")
        b.bgpo_preference_loss(pp, ell[:P], ell[P:], ref[:P], ref[P:], None, None, None, None, None, adv[:P], adv[P:], stats,
                               b.preference_workspace(pp))
        o = oracle.preference_loss(*(t.cpu().numpy() for t in (ell[:P], ell[P:], ref[:P], ref[P:])), mean=True, beta=0.5,
                                   loss_scale=1.0 / P)
        want_adv, want_loss = np.concatenate((o["adv_win"], o["adv_lose"])), o["stats"][0]
    else:
        # exp(B_theta - B_old) A, clipped: d loss / d l_j is the same for every sample of a response
        cp = b.PolicyLoss(B, nt, ratio=b.BGPO_RATIO_SEQUENCE, reduce=b.BGPO_REDUCE_RESPONSES, clip_low=0.1, clip_high=0.1,
                          loss_scale=1.0 / B)
        stats = torch.empty(6, dtype=torch.float64, device="cuda")
        dl = torch.empty_like(ell)
        on = torch.ones(B, nt, dtype=torch.uint8, device="cuda")
        b.bgpo_policy_loss(cp, ell, ref, None, dev["adv"], on, dl, stats, b.policy_workspace(cp))
        adv.copy_(-dl.sum(1))
        s, g, _ = oracle.policy_loss(ell.cpu().numpy(), ref.cpu().numpy(), None, x["adv"], np.ones((B, nt)), ratio="sequence",
                                     reduce="responses", clip_low=0.1, clip_high=0.1, loss_scale=1.0 / B)
        want_adv, want_loss = -g.sum(1), s[0]
        assert 0 < s[5] < s[4]                       # some are clipped, some are not
    assert abs(float(stats[0]) - want_loss) <= 1e-12 * (1 + abs(want_loss))
    assert np.abs(adv.cpu().numpy() - want_adv).max() <= 2.0 ** -23 * np.abs(want_adv).max()
    dX = torch.zeros(B, L, d, device="cuda")
    dW = torch.zeros(d, V, device="cuda")
    e2, g2 = torch.zeros_like(ell), torch.zeros_like(ell)
    loss = torch.zeros(1, dtype=torch.float64, device="cuda")
    nm = torch.zeros(B, nt, dtype=torch.int32, device="cuda")
    b.bgpo_elbo_bwd_accumulate(prob, dev["hidden"], dev["W"], dev["targets"], dev["resp_mask"], adv, None, 1.0, dX, dW, e2, g2,
                               loss, nm, None, None, b.alloc_workspace(prob))
    assert torch.equal(e2, ell)
    norm = torch.empty(1, dtype=torch.float64, device="cuda")
    gl = b.GradList([dX, dW])
    b.bgpo_grad_norm(gl, norm, b.grad_workspace())
    outs = [torch.empty_like(t, dtype=torch.bfloat16) for t in (dX, dW)]
    max_norm = 0.5 * float(norm)
    b.bgpo_grad_clip(gl, max_norm, norm, b.GradList(outs))
    r = elbo.elbo_literal(elbo.Problem(B, L, d, V, nt, seed=w.philox_seed, seq_id_base=w.seq_id_base, bound=1), x["hidden"],
                          x["W"], x["targets"], x["resp_mask"], want_adv, loss_scale=1.0)
    want = oracle.grad_norm([r.dX, r.dW])
    # the ELBO gradients' own bar: 2e-2 of the largest entry
    assert abs(float(norm) - want) <= 2e-2 * want
    for o, t in zip(outs, (r.dX, r.dW)):
        v = t * (max_norm / want)
        assert np.abs(o.double().cpu().numpy() - v).max() <= 2.5e-2 * np.abs(v).max()


def _independent_calls(b, seed):
    """Every operator on inputs, outputs and workspaces of its own; (call, outputs)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, **k: torch.randn(*s, generator=g, device="cuda", **k)  # noqa: E731
    rows, V, B, L, P = 96, 20011, 300, 3001, 64
    f = lambda n, t=torch.float32: torch.empty(n, dtype=t, device="cuda")  # noqa: E731
    x = r(rows, V).bfloat16()
    y = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    logp, ent, lse, a = f(rows), f(rows), f(rows), r(rows)
    dx, lws = torch.empty_like(x), b.logits_workspace(rows, V)
    lp, old, ref, adv = -r(B, L).abs(), -r(B, L).abs(), -r(B, L).abs(), r(B)
    mask = torch.rand(B, L, generator=g, device="cuda") < 0.7
    prob, dl, stats = b.PolicyLoss(B, L, kl_coef=0.1), torch.empty_like(lp), f(6, torch.float64)
    pws = b.policy_workspace(prob)
    pref, dw, dlo, pstats = b.PreferenceLoss(P, L, loss_scale=1 / P), torch.empty_like(lp[:P]), torch.empty_like(lp[:P]), f(3, torch.float64)
    prefws = b.preference_workspace(pref)
    grads, norm, gws = [r(100003), r(77, 501).bfloat16(), r(1 << 20)], f(1, torch.float64), b.grad_workspace()
    outs = [torch.empty_like(t, dtype=torch.bfloat16) for t in grads]
    gl, ol = b.GradList(grads), b.GradList(outs)

    def call(s):
        b.bgpo_logits_logp(x, y, logp, ent, lse, lws, stream=s)
        b.bgpo_logits_logp_bwd(x, y, lse, ent, a, a, dx, stream=s)
        b.bgpo_policy_loss(prob, lp, old, ref, adv, mask, dl, stats, pws, stream=s)
        b.bgpo_preference_loss(pref, lp[:P], lp[P:2 * P], old[:P], old[P:2 * P], mask[:P], mask[P:2 * P], dw, dlo, None, None, None,
                               pstats, prefws, stream=s)
        b.bgpo_grad_norm(gl, norm, gws, stream=s)
        b.bgpo_grad_clip(gl, 3.0, norm, ol, stream=s)

    return call, [logp, ent, lse, dx, dl, stats, dw, dlo, pstats, norm] + outs


def test_calls_on_two_streams_at_once():
    """With workspaces of their own, the bits of calls one after the other."""
    b = lib()
    calls = [_independent_calls(b, seed) for seed in (1, 2)]
    want = []
    for call, outs in calls:
        call(None)
        torch.cuda.synchronize()
        want.append([t.clone() for t in outs])
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        for _, outs in calls:
            for t in outs:
                t.fill_(7.0)
        torch.cuda.synchronize()
        for (call, _), s in zip(calls, streams):
            call(s)
        torch.cuda.synchronize()
        for (_, outs), w in zip(calls, want):
            assert all(torch.equal(t, v) for t, v in zip(outs, w))
