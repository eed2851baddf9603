"""float64 oracle of token log-probabilities, the policy and preference losses
and the gradient norm (numpy; imports nothing from the HIP path).

TEST INFRASTRUCTURE: part of the oracle; see ``oracle/__init__.py``.

Written row by row from the definitions in include/bgpo_policy.h and
include/bgpo_grads.h, without the reorganisations that the kernels make.
"""
import numpy as np


# ---------------------------------------------------------------- logits

def logits_logp(x, targets, row_mask=None, scale=1.0):
    """(logp, entropy, lse), float64 [rows]."""
    x = np.asarray(x, dtype=np.float64)
    out = np.zeros((3, x.shape[0]))
    for r, y in enumerate(targets):
        if y < 0 or (row_mask is not None and not row_mask[r]):
            continue
        z = x[r] * scale
        if np.isnan(z).any() or (z == np.inf).any() or not (z > -np.inf).any():
            out[:, r] = np.nan
            continue
        m = z.max()
        ls = np.log(np.exp(z - m).sum())     # (lse - m, which lse itself may lose)
        lp = z[z > -np.inf] - m - ls
        out[:, r] = z[y] - m - ls if y < len(z) else np.nan, -(np.exp(lp) * lp).sum(), m + ls
    return out


def logits_logp_bwd(x, targets, lse, entropy, dlogp, dentropy=None, row_mask=None, scale=1.0):
    """d (sum_r dlogp_r logp_r + dentropy_r H_r) / d x, with the given statistics."""
    x = np.asarray(x, dtype=np.float64)
    g = np.zeros_like(x)
    for r, y in enumerate(targets):
        a, b = float(dlogp[r]), 0.0 if dentropy is None else float(dentropy[r])
        if y < 0 or (row_mask is not None and not row_mask[r]) or (a == 0 and b == 0):
            continue
        if y >= x.shape[1]:
            g[r] = np.nan
            continue
        lp = x[r] * scale - float(lse[r])
        p = np.exp(lp)
        g[r] = -a * p
        g[r, y] += a
        if b:
            with np.errstate(invalid="ignore"):
                g[r] -= b * np.where(lp == -np.inf, 0.0, p * (lp + float(entropy[r])))
        g[r] *= scale
    return g
