"""Cases of the operators between a policy's log-probabilities and its update.

Five operators of `paper_2510_11683_amd.bgpo`: the log-probability (and
entropy) of a target token in each row of logits, its backward, the clipped
policy loss with a KL term, the preference loss on paired log ratios, and the
norm of many gradients with their clipping.  `run` is one call as a training or
scoring program makes it; without `own` it computes the same in elementary
torch operations.  `exact` restates every quantity in float64.
"""
import math

import torch

own = False

DEV = "cuda"
RATIO = {"token": 0, "sequence": 1}
REDUCE = {"tokens": 0, "responses": 1, "sum": 2}
KL = {"k1": 0, "k2": 1, "k3": 2}
PREF = {"sigmoid": 0, "hinge": 1, "squared": 2}
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32, "f64": torch.float64}


def _logits(name, **kw):
    c = dict(op="logp", rows=8, V=126464, pad=0, dtype="bf16", scale=1.0, masked=0.0, entropy=False, zero_grads=0.0,
             dead_vocab=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _policy(name, **kw):
    c = dict(op="policy", B=8, L=512, pad=0, min_len=0, dtype="f32", ratio="token", reduce="tokens", clip_low=0.2,
             clip_high=0.2, clip_dual=0.0, kl="k3", kl_coef=0.04, adv_per_token=False, noise=0.15)
    c.update(kw)
    return dict(c, name=name) if name else c


def _pref(name, **kw):
    c = dict(op="preference", P=8, L=16, pad=0, min_len=0, masks=False, dtype="f64", kind="sigmoid", reduce="mean",
             beta=0.1, margin=0.0, label_smoothing=0.0, reference=True)
    c.update(kw)
    return dict(c, name=name) if name else c


def _grads(name, **kw):
    c = dict(op="grads", tensors=2, total=1 << 20, largest=0.5, dtype="f32", out="bf16", over=True)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # scoring one new token of each of 8 responses at the vocabulary of the
        # benchmark's head: a serving step, latency and one pass over 2 MB
        _logits("logp_one_token_each", rows=8),
        # the log-probabilities and entropies of a whole batch, 8 responses of 512
        # tokens: prompts and padding are masked, a gigabyte of logits
        _logits("logp_batch", rows=4096, masked=0.2, entropy=True),
        # a reference model with fp32 logits, an odd vocabulary with unused ids
        # (-inf) at its end, rows of odd length, a sampling temperature
        _logits("logp_odd_f32", rows=777, V=32003, pad=2, dtype="f32", scale=1.25, masked=0.3, entropy=True,
                dead_vocab=100),
        # the gradient of the batch's logits: masked rows are cleared, tokens that
        # the clip has cut off have none
        _logits("logp_bwd_batch", op="logp_bwd", rows=4096, masked=0.2, zero_grads=0.1),
        # the same with an entropy bonus, odd sizes, rows that are not aligned
        _logits("logp_bwd_odd", op="logp_bwd", rows=1009, V=50021, masked=0.3, entropy=True, scale=0.8, dead_vocab=21),
        # the objective of one step on 8 responses of 512 tokens (pure latency)
        _policy("policy_step", min_len=128),
        # ELBO estimates of 16 responses, 32 samples each, one ratio per response:
        # the exact ratio's clipped form on what the head's forward returns
        _policy("policy_elbo", B=16, L=32, dtype="f64", ratio="sequence", reduce="responses", kl="k2", kl_coef=0.01,
                noise=0.05),
        # a large batch of long ragged responses, one ratio for each
        _policy("policy_long", B=1024, L=16385, pad=7, min_len=1, ratio="sequence", reduce="responses", clip_low=0.003,
                clip_high=0.004),
        # pairs of responses with their ELBO estimates under both policies
        _pref("preference_elbo"),
        # token log-probabilities of long ragged pairs, summed over each response
        _pref("preference_tokens", P=384, L=8191, pad=1, min_len=1, masks=True, dtype="f32", reduce="sum",
              label_smoothing=0.1),
        # the gradients of a model of 290 tensors, most of them small: norm, and the
        # clipping in place that finds nothing to clip
        _grads("clip_model", tensors=290, total=100_000_001, largest=0.05, dtype="bf16", out="in place", over=False),
        # the gradients of the benchmark's head and hidden states, clipped into the
        # bf16 copies that the optimiser and the predictor's backward take
        _grads("clip_head", tensors=2, total=(8 * 512 + 126464) * 4096, largest=126464 / (8 * 512 + 126464)),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(("logp", "logp_bwd", "policy", "preference", "grads"))
    if op in ("logp", "logp_bwd"):
        dtype = rng.choice(("bf16", "bf16", "f32"))
        V = _log_int(rng, 64, 131071)
        rows = _log_int(rng, 4, max(4, min(8192, (500_000_000 if dtype == "bf16" else 250_000_000) // V)))
        return _logits("", op=op, rows=rows, V=V, pad=rng.choice((0, 0, 1, 3, 8)), dtype=dtype,
                       scale=rng.choice((1.0, 1.0, 0.7, 1.3)), masked=rng.choice((0.0, 0.25)), entropy=rng.random() < 0.5,
                       zero_grads=rng.choice((0.0, 0.15)) if op == "logp_bwd" else 0.0, dead_vocab=rng.randrange(V // 8))
    if op == "policy":
        L = _log_int(rng, 1, 20000)
        B = _log_int(rng, 8, max(8, 16_000_000 // L))
        ratio = rng.choice(("token", "sequence"))
        return _policy("", B=B, L=L, pad=rng.choice((0, 0, 1, 5)), min_len=rng.choice((0, 1)) if L > 1 else 0,
                       dtype=rng.choice(("f32", "f32", "f64")), ratio=ratio, reduce=rng.choice(tuple(REDUCE)),
                       clip_low=rng.choice((0.1, 0.2)), clip_high=rng.choice((0.2, 0.28)), clip_dual=rng.choice((0.0, 3.0)),
                       kl=rng.choice(tuple(KL)), kl_coef=rng.choice((0.0, 0.01, 0.1)),
                       adv_per_token=ratio == "token" and rng.random() < 0.3, noise=rng.choice((0.05, 0.3)))
    if op == "preference":
        L = _log_int(rng, 1, 10000)
        P = _log_int(rng, 1, max(1, min(16384, 3_000_000 // L)))
        kind, masks = rng.choice(tuple(PREF)), rng.random() < 0.6
        return _pref("", P=P, L=L, pad=rng.choice((0, 0, 1, 5)), masks=masks, min_len=1 if masks else 0,
                     dtype=rng.choice(("f32", "f64")), kind=kind, reduce=rng.choice(("sum", "mean")),
                     beta=rng.choice((0.05, 0.1, 0.5)), margin=rng.choice((0.0, 0.3)),
                     label_smoothing=rng.choice((0.0, 0.1)) if kind == "sigmoid" else 0.0, reference=rng.random() < 0.7)
    out = rng.choice(("in place", "bf16", "same"))
    return _grads("", tensors=_log_int(rng, 1, 400), total=_log_int(rng, 2000, 300_000_000),
                  largest=rng.uniform(0.01, 0.9), dtype=rng.choice(("bf16", "f32")), out=out,
                  over=out != "in place" and rng.random() < 0.7)


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) & 0x7FFFFFFFFFFF)


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV, dtype=dtype)


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device=DEV)


def _row_stats(x, scale):
    """(lse, entropy) of scaled rows of logits, float32."""
    lse, ent = [], []
    for part in x.split(512):
        z = part.double() * scale
        l = torch.logsumexp(z, 1)
        lp = z - l[:, None]
        lse.append(l)
        ent.append(-(lp.exp() * lp.clamp_min(-1e30)).sum(1))
    return torch.cat(lse).float(), torch.cat(ent).float()


def _prepare_logits(c, g):
    rows, V, ld = c["rows"], c["V"], c["V"] + c["pad"]
    x = torch.empty(rows, ld, dtype=DTYPE[c["dtype"]], device=DEV)
    for part in x.split(512):
        part.copy_(_randn(g, *part.shape) * 2.5)
    live = V - c["dead_vocab"]
    targets = torch.randint(0, live, (rows,), generator=g, device=DEV, dtype=torch.int32)
    # sampled tokens are likely ones: the target's logit lies near the log-sum-exp
    near = torch.logsumexp(x[:, :live].float() * c["scale"], 1) if rows * V < 1 << 26 else \
        torch.full((rows,), math.log(live) + 3.1 * c["scale"] ** 2, device=DEV)
    x[torch.arange(rows, device=DEV), targets.long()] = ((near - 1.5 * _randn(g, rows).abs()) / c["scale"]).to(x.dtype)
    x[:, live:V] = -math.inf
    mask = None
    if c["masked"]:
        mask = (_rand(g, rows) >= c["masked"]).to(torch.uint8)
        mask[0] = 1
        x[mask == 0] = math.nan                     # what padding holds is nobody's business
    s = dict(x=x[:, :V], targets=targets, mask=mask, scale=c["scale"], op=c["op"])
    f = lambda: torch.empty(rows, dtype=torch.float32, device=DEV)  # noqa: E731
    if c["op"] == "logp":
        s.update(logp=f(), lse=f(), ent=f() if c["entropy"] else None)
        return s
    s["lse"], s["ent"] = _row_stats(s["x"], c["scale"])
    s["dlogp"] = _randn(g, rows) * (_rand(g, rows) >= c["zero_grads"]) / rows
    s["dent"] = torch.full((rows,), -0.01 / rows, device=DEV) * (s["dlogp"] != 0) if c["entropy"] else None
    if not c["entropy"]:
        s["ent"] = None
    s["dx"] = torch.empty_like(x)[:, :V]
    return s


def _lengths(c, g, n):
    """uint8 [n, L + pad] with 1 on the first positions of each row; the first
    row is full, and with min_len 0 every eighth of the others is empty."""
    L = c["L"]
    if not c["min_len"] and c["op"] == "policy" and c["L"] <= 64:
        m = torch.ones(n, L, dtype=torch.uint8, device=DEV)
    else:
        n_i = c["min_len"] + (_rand(g, n) * (L + 1 - c["min_len"])).floor().clamp_max(L - c["min_len"])
        if not c["min_len"]:
            n_i[7::8] = 0
        n_i[0] = L
        m = (torch.arange(L, device=DEV)[None] < n_i[:, None]).to(torch.uint8)
    return torch.nn.functional.pad(m, (0, c["pad"]))


def _prepare_policy(c, g):
    B, L, ld, t = c["B"], c["L"], c["L"] + c["pad"], DTYPE[c["dtype"]]
    mask = _lengths(c, g, B)
    level = -30.0 if c["dtype"] == "f64" else -1.5
    old = level * _rand(g, B, ld).to(t)
    logp = old + c["noise"] * _randn(g, B, ld, dtype=t)
    ref = logp + c["noise"] * _randn(g, B, ld, dtype=t)
    logp[mask == 0] = math.nan
    adv = _randn(g, B, ld) if c["adv_per_token"] else _randn(g, B)
    return dict(op="policy", c=c, logp=logp[:, :L], old=old[:, :L], ref=ref[:, :L], mask=mask[:, :L],
                adv=adv[:, :L] if c["adv_per_token"] else adv, dlogp=torch.empty(B, ld, dtype=t, device=DEV)[:, :L],
                stats=torch.empty(6, dtype=torch.float64, device=DEV))


def _prepare_pref(c, g):
    P, L, ld, t = c["P"], c["L"], c["L"] + c["pad"], DTYPE[c["dtype"]]
    s = dict(op="preference", c=c)
    for k in ("win", "lose"):
        s[k] = (-2.0 * _rand(g, P, ld).to(t))[:, :L]
        s[k + "_ref"] = (s[k] + 0.3 * _randn(g, P, L, dtype=t)).contiguous() if not c["pad"] else None
        if c["pad"]:
            s[k + "_ref"] = torch.nn.functional.pad(s[k] + 0.3 * _randn(g, P, L, dtype=t), (0, c["pad"]))[:, :L]
        if not c["reference"]:
            s[k + "_ref"] = None
        s[k + "_mask"] = _lengths(c, g, P)[:, :L] if c["masks"] else None
        s["d" + k] = torch.empty(P, ld, dtype=t, device=DEV)[:, :L]
        s["adv_" + k] = torch.empty(P, dtype=torch.float32, device=DEV)
    s["margins"] = torch.empty(P, dtype=torch.float64, device=DEV)
    s["stats"] = torch.empty(3, dtype=torch.float64, device=DEV)
    return s


def _sizes(c):
    """Element counts of the list: the largest takes its share, the others fall
    off geometrically, none below one."""
    n, total = c["tensors"], c["total"]
    if n == 1:
        return [total]
    first = max(1, int(total * c["largest"]))
    if n == 2:
        return [first, max(1, total - first)]
    w = [math.exp(-5.0 * ((i * 7919) % n) / n) for i in range(n - 1)]
    k = (total - first) / sum(w)
    return [first] + [max(1, int(k * v)) for v in w]


def _prepare_grads(c, g):
    sizes, t = _sizes(c), DTYPE[c["dtype"]]
    flat = torch.empty(sum(sizes), dtype=t, device=DEV)
    for part in flat.split(1 << 26):
        part.copy_(_randn(g, part.numel()))
    rms = 1e-3
    flat *= rms
    norm = rms * math.sqrt(flat.numel())             # about the norm
    ot = {"in place": None, "same": t, "bf16": torch.bfloat16}[c["out"]]
    dst = None if ot is None else torch.empty(flat.numel(), dtype=ot, device=DEV)
    return dict(op="grads", flat=flat, tensors=list(flat.split(sizes)), dst=dst,
                outs=None if dst is None else list(dst.split(sizes)), max_norm=norm * (0.4 if c["over"] else 2.0),
                norm=torch.empty(1, dtype=torch.float64, device=DEV))


def prepare(case, seed):
    g = _gen(seed)
    if case["op"] in ("logp", "logp_bwd"):
        return _prepare_logits(case, g)
    return {"policy": _prepare_policy, "preference": _prepare_pref, "grads": _prepare_grads}[case["op"]](case, g)


# ---------------------------------------------------------------- the framework's calls

def _own_scale(c):
    """The scale as the plain form weighs with it: a sum's is a number of 32 bits there."""
    scale = _policy_scale(c)
    return float(torch.tensor(scale, dtype=torch.float32)) if c["reduce"] == "sum" else scale


def _own(s):
    from paper_2510_11683_amd import bgpo
    if s["op"] == "logp":
        if "ws" not in s:
            s["ws"] = bgpo.logits_workspace(*s["x"].shape)
        bgpo.bgpo_logits_logp(s["x"], s["targets"], s["logp"], s["ent"], s["lse"], s["ws"], row_mask=s["mask"],
                              scale=s["scale"])
        return [s["logp"], s["lse"]] + ([s["ent"]] if s["ent"] is not None else [])
    if s["op"] == "logp_bwd":
        bgpo.bgpo_logits_logp_bwd(s["x"], s["targets"], s["lse"], s["ent"], s["dlogp"], s["dent"], s["dx"],
                                  row_mask=s["mask"], scale=s["scale"])
        return s["dx"]
    if s["op"] == "policy":
        c = s["c"]
        if "ws" not in s:
            s["prob"] = bgpo.PolicyLoss(c["B"], c["L"], ratio=RATIO[c["ratio"]], reduce=REDUCE[c["reduce"]], kl=KL[c["kl"]],
                                        clip_low=c["clip_low"], clip_high=c["clip_high"], clip_dual=c["clip_dual"],
                                        kl_coef=c["kl_coef"], loss_scale=_own_scale(c))
            s["ws"] = bgpo.policy_workspace(s["prob"])
        bgpo.bgpo_policy_loss(s["prob"], s["logp"], s["old"], s["ref"], s["adv"], s["mask"], s["dlogp"], s["stats"], s["ws"])
        return [s["stats"][:4], s["stats"][4:], s["dlogp"]]
    if s["op"] == "preference":
        c = s["c"]
        if "ws" not in s:
            s["prob"] = bgpo.PreferenceLoss(c["P"], c["L"], kind=PREF[c["kind"]], mean=c["reduce"] == "mean", beta=c["beta"],
                                            margin=c["margin"], label_smoothing=c["label_smoothing"], loss_scale=1.0 / c["P"])
            s["ws"] = bgpo.preference_workspace(s["prob"])
        bgpo.bgpo_preference_loss(s["prob"], s["win"], s["lose"], s["win_ref"], s["lose_ref"], s["win_mask"], s["lose_mask"],
                                  s["dwin"], s["dlose"], s["margins"], s["adv_win"], s["adv_lose"], s["stats"], s["ws"])
        return [s["stats"][:1], s["stats"][1:], s["margins"], s["adv_win"], s["adv_lose"], s["dwin"], s["dlose"]]
    if "ws" not in s:
        s["ws"] = bgpo.grad_workspace()
        s["list"] = bgpo.GradList(s["tensors"])
        s["list_out"] = None if s["outs"] is None else bgpo.GradList(s["outs"])
    bgpo.bgpo_grad_norm(s["list"], s["norm"], s["ws"])
    bgpo.bgpo_grad_clip(s["list"], s["max_norm"], s["norm"], s["list_out"])
    return [s["norm"], s["flat"] if s["dst"] is None else s["dst"]]


# ---------------------------------------------------------------- the plain forms

def _policy_scale(c):
    """The mean over the batch: over its tokens or its responses."""
    return 1.0 if c["reduce"] == "tokens" else 1.0 / c["B"] if c["reduce"] == "responses" else 1.0 / (c["B"] * c["L"])


def _plain_logp(s):
    live = None if s["mask"] is None else s["mask"] != 0
    z = s["x"].float() * s["scale"]
    m = z.amax(1, keepdim=True)
    t = z - m
    e = torch.exp(t)
    sums = e.sum(1)
    logs = torch.log(sums)
    lse = m[:, 0] + logs
    logp = t.gather(1, s["targets"].long()[:, None])[:, 0] - logs
    out = [logp, lse]
    if s["ent"] is not None:
        out.append(logs - torch.where(e > 0, e * t, 0.0).sum(1) / sums)
    return out if live is None else [torch.where(live, v, 0.0) for v in out]


def _plain_logp_bwd(s):
    live = s["dlogp"] != 0
    if s["dent"] is not None:
        live = live | (s["dent"] != 0)
    if s["mask"] is not None:
        live = live & (s["mask"] != 0)
    t = s["x"].float() * s["scale"] - s["lse"][:, None]
    p = torch.exp(t)
    g = -p * s["dlogp"][:, None]
    if s["dent"] is not None:
        g = g - torch.where(p > 0, p * (t + s["ent"][:, None]), 0.0) * s["dent"][:, None]
    y = s["targets"].long()[:, None]
    g.scatter_add_(1, y, s["dlogp"][:, None])
    return torch.where(live[:, None], g * s["scale"], 0.0).to(s["x"].dtype)


def _plain_policy(s):
    c, t = s["c"], s["logp"].dtype
    on = s["mask"] != 0
    n = on.sum(1, keepdim=True).double()
    total = n.sum()
    d = torch.where(on, s["logp"].double() - s["old"].double(), 0.0)
    q = torch.where(on, s["ref"].double() - s["logp"].double(), 0.0)
    adv = s["adv"].double() if c["adv_per_token"] else s["adv"].double()[:, None]
    if c["ratio"] == "sequence":
        x = d.sum(1, keepdim=True) / n.clamp_min(1.0)
        r = torch.exp(x)
    else:
        r = torch.exp(d)
    lo, hi = 1.0 - c["clip_low"], 1.0 + c["clip_high"]
    free, held = r * adv, r.clamp(lo, hi) * adv
    obj = torch.minimum(free, held)
    cut = held < free
    if c["clip_dual"]:
        dual = (adv < 0) & (c["clip_dual"] * adv > obj)
        obj, cut = torch.where(dual, c["clip_dual"] * adv, obj), cut | dual
    w = _policy_scale(c) / (total if c["reduce"] == "tokens" else n.clamp_min(1.0) if c["reduce"] == "responses" else 1.0)
    w = torch.where(on, w, 0.0)
    dpg = torch.where(cut, 0.0, -r * adv)
    if c["ratio"] == "sequence":
        # every token of a response moves its one ratio by 1 / n
        dl = torch.where(on, dpg * w.sum(1, keepdim=True) / n.clamp_min(1.0), 0.0)
    else:
        dl = dpg * w
    if c["kl"] == "k1":
        kl, dkl = -q, torch.ones_like(q)
    elif c["kl"] == "k2":
        kl, dkl = 0.5 * q * q, -q
    else:
        kl, dkl = torch.expm1(q) - q, -torch.expm1(q)
    policy, klsum = -(w * obj).sum(), (w * kl).sum()
    dl = dl + c["kl_coef"] * w * dkl
    cuts = (cut & on).sum().double()
    stats = torch.stack((policy + c["kl_coef"] * klsum, policy, klsum, (w * d).sum(), total, cuts))
    return [stats[:4], stats[4:], torch.where(on, dl, 0.0).to(t)]


def _plain_pref(s):
    c = s["c"]

    def estimate(k):
        v = s[k].double() if s[k + "_ref"] is None else s[k].double() - s[k + "_ref"].double()
        if s[k + "_mask"] is not None:
            v = torch.where(s[k + "_mask"] != 0, v, 0.0)
            n = (s[k + "_mask"] != 0).sum(1).double()
        else:
            n = torch.full((c["P"],), float(c["L"]), dtype=torch.float64, device=DEV)
        div = n.clamp_min(1.0) if c["reduce"] == "mean" else torch.ones_like(n)
        return v.sum(1) / div, div

    (sw, nw), (sl, nl) = estimate("win"), estimate("lose")
    m = c["beta"] * (sw - sl) - c["margin"]
    if c["kind"] == "sigmoid":
        e = c["label_smoothing"]
        softplus = lambda v: v.clamp_min(0.0) + torch.log1p(torch.exp(-v.abs()))  # noqa: E731
        loss = (1 - e) * softplus(-m) + e * softplus(m)
        dm = -(1 - e) / (1 + torch.exp(m)) + e / (1 + torch.exp(-m))
    elif c["kind"] == "hinge":
        loss, dm = (1 - m).clamp_min(0.0), torch.where(m < 1, -1.0, 0.0).double()
    else:
        loss, dm = ((m - 0.5) / c["beta"]) ** 2, 2 * (m - 0.5) / c["beta"] ** 2
    k = dm * c["beta"] / c["P"]

    def spread(v, name):
        g = v[:, None].expand(c["P"], c["L"])
        if s[name + "_mask"] is not None:
            g = torch.where(s[name + "_mask"] != 0, g, 0.0)
        return g.to(s[name].dtype)

    stats = torch.stack((loss.sum() / c["P"], (m > 0).sum().double(), m.sum()))
    return [stats[:1], stats[1:], m, -k.float(), k.float(), spread(k / nw, "win"), spread(-k / nl, "lose")]


def _plain_grads(s):
    norm = torch.stack([t.double().square().sum() for t in s["tensors"]]).sum().sqrt()
    coef = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0).float()
    if s["dst"] is None:
        [t.copy_(t.float() * coef) for t in s["tensors"]]
        return [norm.reshape(1), s["flat"]]
    [o.copy_(t.float() * coef) for t, o in zip(s["tensors"], s["outs"])]
    return [norm.reshape(1), s["dst"]]


def run(state):
    if own:
        return _own(state)
    return {"logp": _plain_logp, "logp_bwd": _plain_logp_bwd, "policy": _plain_policy, "preference": _plain_pref,
            "grads": _plain_grads}[state["op"]](state)


# ---------------------------------------------------------------- float64

def _exact_logits(c, s):
    x, y, rows = s["x"], s["targets"].long(), c["rows"]
    live = torch.ones(rows, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"].bool()
    at = live.nonzero()[:, 0]
    f = lambda: torch.zeros(rows, dtype=torch.float64, device=DEV)  # noqa: E731
    if c["op"] == "logp":
        logp, lse, ent = f(), f(), f()
        for k in at.split(256):
            z = x[k].double() * s["scale"]
            lp = torch.log_softmax(z, 1)
            logp[k] = lp.gather(1, y[k, None])[:, 0]
            lse[k] = torch.logsumexp(z, 1)
            ent[k] = torch.special.entr(lp.exp()).sum(1)
        return [logp, lse] + ([ent] if c["entropy"] else [])
    dx = torch.zeros(rows, c["V"], dtype=torch.float64, device=DEV)
    for k in at.split(256):
        z = x[k].double() * s["scale"]
        lp = z - s["lse"][k, None].double()
        p = lp.exp()
        a = s["dlogp"][k, None].double()
        one = torch.zeros_like(p).scatter_(1, y[k, None], 1.0)
        d = a * (one - p)
        if c["entropy"]:
            b = s["dent"][k, None].double()
            d = d + b * (torch.special.entr(p) - p * s["ent"][k, None].double())
        dx[k] = d * s["scale"]
    return dx


def _exact_policy(c, s):
    """Through autograd, from the objective as it is written."""
    on = s["mask"].bool()
    n = on.sum(1).double()
    lp = torch.where(on, s["logp"].double(), 0.0).requires_grad_(True)
    zero = torch.zeros((), dtype=torch.float64, device=DEV)
    d = torch.where(on, lp - s["old"].double(), zero)
    adv = s["adv"].double() if c["adv_per_token"] else s["adv"].double()[:, None].expand(-1, c["L"])
    some = torch.where(n > 0, n, 1.0)
    x = (d.sum(1) / some)[:, None].expand(-1, c["L"]) if c["ratio"] == "sequence" else d
    lo, hi = math.log(1.0 - c["clip_low"]), math.log(1.0 + c["clip_high"])
    up = x.clamp_max(hi).exp() * adv                          # a gain is held from above
    down = x.clamp_min(lo).exp() * adv                        # a loss from below
    if c["clip_dual"]:
        down = x.clamp(lo, math.log(c["clip_dual"])).exp() * adv
    obj = torch.where(adv >= 0, up, down)
    cut = torch.where(adv >= 0, x > hi, x < lo) & (adv != 0)
    if c["clip_dual"]:
        cut = cut | ((adv < 0) & (x > math.log(c["clip_dual"])))
    scale = _policy_scale(c)
    if c["reduce"] == "tokens":
        w = on.double() * (scale / n.sum())
    elif c["reduce"] == "responses":
        w = on.double() * (scale / some)[:, None]
    else:
        w = on.double() * scale
    q = torch.where(on, s["ref"].double() - lp, zero)
    kl = {"k1": -q, "k2": q.square() / 2, "k3": torch.special.expm1(q) - q}[c["kl"]]
    policy, klsum = -(w * obj).sum(), (w * kl).sum()
    loss = policy + c["kl_coef"] * klsum
    (dl,) = torch.autograd.grad(loss, lp)
    stats = torch.stack((loss, policy, klsum, (w * d).sum(), n.sum(), (cut & on).sum().double()))
    stats = stats.detach()
    return [stats[:4], stats[4:], dl.detach()]


def _exact_pref(c, s):
    """Through autograd, from the loss as it is written."""
    leaf, score = {}, {}
    for k in ("win", "lose"):
        on = torch.ones(c["P"], c["L"], dtype=torch.bool, device=DEV) if s[k + "_mask"] is None else s[k + "_mask"].bool()
        leaf[k] = s[k].double().requires_grad_(True)
        v = leaf[k] - (0.0 if s[k + "_ref"] is None else s[k + "_ref"].double())
        score[k] = (v * on).sum(1) / (on.sum(1) if c["reduce"] == "mean" else 1)
        score[k].retain_grad()
    m = c["beta"] * (score["win"] - score["lose"]) - c["margin"]
    e = c["label_smoothing"]
    if c["kind"] == "sigmoid":
        loss = -(1 - e) * torch.nn.functional.logsigmoid(m) - e * torch.nn.functional.logsigmoid(-m)
    elif c["kind"] == "hinge":
        loss = torch.relu(1 - m)
    else:
        loss = ((m - 0.5) / c["beta"]).square()
    total = loss.mean()
    total.backward()
    stats = torch.stack((total.detach(), (m > 0).sum().double(), m.detach().sum()))
    return [stats[:1], stats[1:], m.detach(), -score["win"].grad, -score["lose"].grad, leaf["win"].grad, leaf["lose"].grad]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("logp", "logp_bwd"):
        return _exact_logits(case, s)
    if case["op"] == "policy":
        return _exact_policy(case, s)
    if case["op"] == "preference":
        return _exact_pref(case, s)
    sq = 0.0
    for part in s["flat"].split(1 << 26):
        sq += float(torch.dot(part.double(), part.double()))
    norm = math.sqrt(sq)
    coef = min(1.0, s["max_norm"] / norm)
    return [torch.tensor([norm], dtype=torch.float64), s["flat"].double() * coef]


# ---------------------------------------------------------------- work

def work(case):
    c = case
    if c["op"] in ("logp", "logp_bwd"):
        e = 2 if c["dtype"] == "bf16" else 4
        live = c["rows"] * (1 - c["masked"])
        n = live * c["V"]
        if c["op"] == "logp":
            return {"bytes": e * n + 4.0 * live + c["rows"] * (12.0 if c["entropy"] else 8.0), "flops": 5.0 * n}
        n *= 1 - c["zero_grads"]
        return {"bytes": e * (n + c["rows"] * c["V"]) + 12.0 * c["rows"], "flops": 5.0 * n}
    e = {"bf16": 2, "f32": 4, "f64": 8}[c["dtype"]]
    if c["op"] == "policy":
        n = c["B"] * c["L"]
        share = 0.5 if c["min_len"] or c["L"] > 64 else 1.0       # mean length of ragged rows
        if c["min_len"] > 1:
            share = (c["min_len"] / c["L"] + 1) / 2
        adv = 4.0 * n * share if c["adv_per_token"] else 4.0 * c["B"]
        return {"bytes": n * (1.0 + e) + 3.0 * e * n * share + adv, "flops": 60.0 * n * share}
    if c["op"] == "preference":
        n = 2.0 * c["P"] * c["L"]
        share = 0.5 if c["masks"] else 1.0
        return {"bytes": n * e + n * share * e * (2 if c["reference"] else 1) + (n if c["masks"] else 0) + 16.0 * c["P"],
                "flops": 4.0 * n * share + 100.0 * c["P"]}
    n = sum(_sizes(c))
    o = 0 if c["out"] == "in place" else 2 if c["out"] == "bf16" else e
    return {"bytes": float(n) * (e + o) + 8.0, "flops": (2.0 if o == 0 else 3.0) * n}
