"""What the log-probability, loss and gradient entry points refuse, on the host
before any HIP call (no GPU; the pointers are never followed), and what the
binding refuses before the library is reached."""
import ctypes
import math
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2510_11683_amd", "libbgpo.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libbgpo.so not built")

INVALID, WORKSPACE, UNSUPPORTED = -1, -2, -4


@pytest.fixture(scope="module")
def b():
    from paper_2510_11683_amd import bgpo
    return bgpo


def test_exports_what_the_headers_declare(b):
    names = set()
    for h in ("bgpo_policy.h", "bgpo_grads.h"):
        src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", h)).read(), flags=re.S)
        names |= set(re.findall(r"\b(bgpo_\w+)\s*\(", src))
    assert {"bgpo_logits_logp", "bgpo_policy_loss", "bgpo_preference_loss", "bgpo_grad_norm", "bgpo_grad_clip"} <= names
    for n in names:
        assert hasattr(b._lib, n), n


def at(k):
    """An address of its own, far from every other."""
    return ctypes.c_void_p((k + 1) << 44)


def _logits(b, **kw):
    f = dict(rows=4, ld=128, V=100, in_dtype=0, scale=1.0, reserved=0)
    f.update(kw)
    return b._Logits(**f)


def _logp(b, prob, over=()):
    args = [at(0), at(1), at(2), at(3), at(4), at(5), at(6), 1 << 30, None]
    for i, v in dict(over).items():
        args[i] = v
    return b._lib.bgpo_logits_logp(ctypes.byref(prob) if prob is not None else None, *args)


def _logp_bwd(b, prob, over=()):
    args = [at(0), at(1), at(2), at(3), at(4), at(5), at(6), at(7), 128, None]
    for i, v in dict(over).items():
        args[i] = v
    return b._lib.bgpo_logits_logp_bwd(ctypes.byref(prob) if prob is not None else None, *args)


BAD_LOGITS = [(dict(rows=-1), INVALID), (dict(V=0), INVALID), (dict(V=-5), INVALID), (dict(ld=99), INVALID),
              (dict(in_dtype=2), INVALID), (dict(in_dtype=-1), INVALID), (dict(scale=0.0), INVALID),
              (dict(scale=-1.0), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID), (dict(scale=2.0 ** 65), UNSUPPORTED),
              (dict(reserved=1), INVALID), (dict(rows=1 << 31), UNSUPPORTED),
              (dict(V=(1 << 24) + 1, ld=1 << 25), UNSUPPORTED), (dict(ld=(1 << 54) + 1), INVALID)]


@pytest.mark.parametrize("kw,status", BAD_LOGITS)
def test_logits_problems(b, kw, status):
    n = ctypes.c_size_t(0)
    p = _logits(b, **kw)
    if "ld" not in kw or "V" in kw:
        assert b._lib.bgpo_logits_workspace_size(ctypes.byref(p), ctypes.byref(n)) == status
    assert _logp(b, p) == status
    assert _logp_bwd(b, p) == status


def test_logits_pointers(b):
    assert b._lib.bgpo_logits_workspace_size(None, ctypes.byref(ctypes.c_size_t(0))) == INVALID
    assert b._lib.bgpo_logits_workspace_size(ctypes.byref(_logits(b)), None) == INVALID
    assert _logp(b, None) == INVALID and _logp_bwd(b, None) == INVALID
    for i in (0, 1, 3):
        assert _logp(b, _logits(b), {i: None}) == INVALID
    for i in (0, 1, 3, 5, 7):
        assert _logp_bwd(b, _logits(b), {i: None}) == INVALID
    assert _logp_bwd(b, _logits(b), {4: None}) == INVALID           # dentropy without the entropy
    # alignment to the element types
    off = lambda k, n: ctypes.c_void_p(at(k).value + n)  # noqa: E731
    for i, n in ((0, 1), (1, 2), (3, 2), (4, 1), (5, 2)):
        assert _logp(b, _logits(b), {i: off(i, n)}) == INVALID
    for i, n in ((0, 1), (1, 2), (3, 2), (4, 2), (5, 2), (6, 2), (7, 1)):
        assert _logp_bwd(b, _logits(b), {i: off(i, n)}) == INVALID
    assert _logp(b, _logits(b, in_dtype=1), {0: off(0, 2)}) == INVALID
    assert _logp_bwd(b, _logits(b), {8: 99}) == INVALID             # rows of the gradient overlap
    # outputs over inputs and over each other (the last byte of 4 rows counts)
    last = at(0).value + 2 * (3 * 128 + 100)
    assert _logp(b, _logits(b), {3: ctypes.c_void_p(last - 4)}) == INVALID
    assert _logp(b, _logits(b), {4: off(3, 12)}) == INVALID
    assert _logp(b, _logits(b), {5: at(1)}) == INVALID
    assert _logp_bwd(b, _logits(b), {7: off(0, 2)}) == INVALID      # in place, but shifted
    assert _logp_bwd(b, _logits(b, ld=130), {7: at(0)}) == INVALID  # in place, another stride
    assert _logp_bwd(b, _logits(b), {7: off(5, 8)}) == INVALID


def test_empty_batches_of_logits_are_done(b):
    p = _logits(b, rows=0)
    assert _logp(b, p, {i: None for i in range(6)}) == 0
    assert _logp_bwd(b, p, {i: None for i in range(8)}) == 0


# ---------------------------------------------------------------- policy loss

def _policy(b, B=4, L=100, ld=(128,) * 5 + (0,), dtype=1, **kw):
    p = b.PolicyLoss(B, L).c(ld, dtype)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _policy_loss(b, prob, over=()):
    # logp, old, ref, adv, mask, dlogp, stats, flags, workspace
    args = [at(k) for k in range(9)] + [1 << 30, None]
    for i, v in dict(over).items():
        args[i] = v
    return b._lib.bgpo_policy_loss(ctypes.byref(prob) if prob is not None else None, *args)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), INVALID), (dict(L=0), INVALID), (dict(L=-3), INVALID), (dict(dtype=0), INVALID), (dict(dtype=3), INVALID),
    (dict(ratio=2), INVALID), (dict(ratio=-1), INVALID), (dict(reduce=3), INVALID), (dict(reduce=-1), INVALID),
    (dict(kl=3), INVALID), (dict(kl=-1), INVALID), (dict(clip_low=-0.1), INVALID), (dict(clip_low=1.1), INVALID),
    (dict(clip_low=math.nan), INVALID), (dict(clip_high=-0.1), INVALID), (dict(clip_high=math.nan), INVALID),
    (dict(clip_dual=1.0), INVALID), (dict(clip_dual=-2.0), INVALID), (dict(clip_dual=math.inf), INVALID),
    (dict(kl_coef=math.nan), INVALID), (dict(loss_scale=math.inf), INVALID), (dict(ld_adv=-1), INVALID),
    (dict(ratio=1, ld_adv=128), INVALID), (dict(B=1 << 21, L=1 << 20), UNSUPPORTED), (dict(B=1, L=(1 << 30) + 1), UNSUPPORTED)])
def test_policy_problems(b, kw, status):
    n = ctypes.c_size_t(0)
    p = _policy(b, **kw)
    assert b._lib.bgpo_policy_workspace_size(ctypes.byref(p), ctypes.byref(n)) == status
    assert _policy_loss(b, p) == status


def test_policy_pointers(b):
    n = ctypes.c_size_t(0)
    assert b._lib.bgpo_policy_workspace_size(None, ctypes.byref(n)) == INVALID
    assert b._lib.bgpo_policy_workspace_size(ctypes.byref(_policy(b)), None) == INVALID
    assert b._lib.bgpo_policy_workspace_size(ctypes.byref(_policy(b)), ctypes.byref(n)) == 0
    assert _policy_loss(b, None) == INVALID
    for i in (0, 3, 4, 6):
        assert _policy_loss(b, _policy(b), {i: None}) == INVALID
    assert _policy_loss(b, _policy(b, kl_coef=0.1), {2: None}) == INVALID       # a KL term without a reference
    for k in ("ld_logp", "ld_old", "ld_ref", "ld_mask", "ld_dlogp", "ld_adv"):
        assert _policy_loss(b, _policy(b, **{k: 99})) == INVALID
        assert _policy_loss(b, _policy(b, **{k: 1 << 55})) == INVALID
    off = lambda k, m: ctypes.c_void_p(at(k).value + m)  # noqa: E731
    for i in (0, 1, 2, 3, 5, 7):
        assert _policy_loss(b, _policy(b), {i: off(i, 2)}) == INVALID
    assert _policy_loss(b, _policy(b), {6: off(6, 4)}) == INVALID
    for i in (0, 1, 2, 5):
        assert _policy_loss(b, _policy(b, dtype=2), {i: off(i, 4)}) == INVALID
    # the gradient in place of an input; the statistics in the last row's last bytes
    for i in (0, 1, 2, 4):
        assert _policy_loss(b, _policy(b), {5: at(i)}) == INVALID
    assert _policy_loss(b, _policy(b), {5: at(3)}) == INVALID
    assert _policy_loss(b, _policy(b), {6: off(0, 4 * (3 * 128 + 100) - 8)}) == INVALID
    assert _policy_loss(b, _policy(b), {7: off(6, 40)}) == INVALID
    for i, v in ((8, None), (8, off(8, 128)), (9, n.value - 1)):
        assert _policy_loss(b, _policy(b), {i: v}) == WORKSPACE


# ---------------------------------------------------------------- preference loss

def _pref(b, P=4, L=100, ld=(128,) * 8 + (1,), dtype=1, **kw):
    p = b.PreferenceLoss(P, L).c(ld, dtype)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _pref_loss(b, prob, over=()):
    # win, lose, their references, masks, gradients, margins, advantages, stats, flags, workspace
    args = [at(k) for k in range(14)] + [1 << 30, None]
    for i, v in dict(over).items():
        args[i] = v
    return b._lib.bgpo_preference_loss(ctypes.byref(prob) if prob is not None else None, *args)


@pytest.mark.parametrize("kw,status", [
    (dict(P=0), INVALID), (dict(L=0), INVALID), (dict(dtype=0), INVALID), (dict(dtype=3), INVALID), (dict(kind=3), INVALID),
    (dict(kind=-1), INVALID), (dict(mean=2), INVALID), (dict(mean=-1), INVALID), (dict(reserved=1), INVALID),
    (dict(beta=0.0), INVALID), (dict(beta=-1.0), INVALID), (dict(beta=math.inf), INVALID), (dict(beta=math.nan), INVALID),
    (dict(margin=math.nan), INVALID), (dict(loss_scale=math.inf), INVALID), (dict(label_smoothing=-0.1), INVALID),
    (dict(label_smoothing=1.0), INVALID), (dict(label_smoothing=0.1, kind=1), INVALID),
    (dict(P=1 << 20, L=1 << 20), UNSUPPORTED), (dict(P=1, L=(1 << 30) + 1), UNSUPPORTED)])
def test_preference_problems(b, kw, status):
    n = ctypes.c_size_t(0)
    p = _pref(b, **kw)
    assert b._lib.bgpo_preference_workspace_size(ctypes.byref(p), ctypes.byref(n)) == status
    assert _pref_loss(b, p) == status


def test_preference_pointers(b):
    n = ctypes.c_size_t(0)
    assert b._lib.bgpo_preference_workspace_size(None, ctypes.byref(n)) == INVALID
    assert b._lib.bgpo_preference_workspace_size(ctypes.byref(_pref(b)), None) == INVALID
    assert b._lib.bgpo_preference_workspace_size(ctypes.byref(_pref(b)), ctypes.byref(n)) == 0
    assert _pref_loss(b, None) == INVALID
    for i in (0, 1, 2, 3, 4, 5, 6, 7, 9, 10, 11):
        assert _pref_loss(b, _pref(b), {i: None}) == INVALID
    for k in ("ld_win", "ld_lose", "ld_win_ref", "ld_lose_ref", "ld_win_mask", "ld_lose_mask", "ld_dwin", "ld_dlose"):
        assert _pref_loss(b, _pref(b, **{k: 99})) == INVALID
    assert _pref_loss(b, _pref(b, adv_stride=0)) == INVALID
    off = lambda k, m: ctypes.c_void_p(at(k).value + m)  # noqa: E731
    for i in (0, 1, 2, 3, 6, 7, 9, 10, 12):
        assert _pref_loss(b, _pref(b), {i: off(i, 2)}) == INVALID
    for i in (8, 11):
        assert _pref_loss(b, _pref(b), {i: off(i, 4)}) == INVALID
    for out in (6, 7):
        for i in range(6):
            assert _pref_loss(b, _pref(b), {out: at(i)}) == INVALID
    assert _pref_loss(b, _pref(b), {7: off(6, 4 * 50)}) == INVALID              # rows of the gradients overlap
    assert _pref_loss(b, _pref(b, ld_dwin=256, ld_dlose=256), {7: off(6, 4 * 99)}) == INVALID
    assert _pref_loss(b, _pref(b, ld_dwin=256, ld_dlose=256), {7: off(6, 4 * 157)}) == INVALID
    assert _pref_loss(b, _pref(b), {10: at(9)}) == INVALID
    assert _pref_loss(b, _pref(b, adv_stride=2), {10: off(9, 8)}) == INVALID
    assert _pref_loss(b, _pref(b), {11: off(8, 24)}) == INVALID
    # what interleaves without sharing a byte gets as far as the workspace
    ok = {13: None}
    assert _pref_loss(b, _pref(b, ld_dwin=256, ld_dlose=256), {7: off(6, 4 * 100), **ok}) == WORKSPACE
    assert _pref_loss(b, _pref(b, ld_dwin=256, ld_dlose=256), {6: off(7, 4 * 156), **ok}) == WORKSPACE
    assert _pref_loss(b, _pref(b, adv_stride=2), {10: off(9, 4), **ok}) == WORKSPACE
    for i, v in ((13, None), (13, off(13, 128)), (14, n.value - 1)):
        assert _pref_loss(b, _pref(b), {i: v}) == WORKSPACE


# ---------------------------------------------------------------- gradients

def _list(b, *entries):
    return (b._Tensor * max(1, len(entries)))(*[b._Tensor(*e) for e in entries])


BAD_ENTRIES = [((1 << 44, -1, 1, 0), INVALID), ((None, 4, 1, 0), INVALID), ((1 << 44, 4, 2, 0), INVALID),
               ((1 << 44, 4, -1, 0), INVALID), ((1 << 44, 4, 1, 1), INVALID), (((1 << 44) + 2, 4, 1, 0), INVALID),
               (((1 << 44) + 1, 4, 0, 0), INVALID), ((1 << 44, (1 << 38) + 1, 1, 0), UNSUPPORTED), ((1 << 48, 4, 1, 0), UNSUPPORTED)]


@pytest.mark.parametrize("entry,status", BAD_ENTRIES)
def test_gradient_entries(b, entry, status):
    g = _list(b, (1 << 45, 8, 1, 0), entry)
    n = b._lib.bgpo_grad_workspace_size()
    assert b._lib.bgpo_grad_norm(g, 2, 0, at(3), None, at(4), n, None) == status
    assert b._lib.bgpo_grad_clip(g, None, 2, 1.0, at(3), None) == status
    ok = _list(b, (1 << 46, 8, 1, 0), (1 << 47, 4, 1, 0))
    assert b._lib.bgpo_grad_clip(ok, g, 2, 1.0, at(3), None) == status


def test_gradient_arguments(b):
    g = _list(b, (1 << 45, 8, 1, 0), (1 << 46, 8, 0, 0))
    n = b._lib.bgpo_grad_workspace_size()
    norm = b._lib.bgpo_grad_norm
    assert norm(None, 2, 0, at(3), None, at(4), n, None) == INVALID
    assert norm(g, -1, 0, at(3), None, at(4), n, None) == INVALID
    for kind in (-1, 2):
        assert norm(g, 2, kind, at(3), None, at(4), n, None) == INVALID
    assert norm(g, 2, 0, None, None, at(4), n, None) == INVALID
    assert norm(g, 2, 0, ctypes.c_void_p(at(3).value + 4), None, at(4), n, None) == INVALID
    assert norm(g, 2, 0, at(3), ctypes.c_void_p(at(5).value + 2), at(4), n, None) == INVALID
    assert norm(g, 2, 0, at(3), None, None, n, None) == WORKSPACE
    assert norm(g, 2, 0, at(3), None, at(4), n - 1, None) == WORKSPACE
    assert norm(g, 2, 0, at(3), None, ctypes.c_void_p(at(4).value + 4), n, None) == WORKSPACE
    clip = b._lib.bgpo_grad_clip
    for bad in (-1.0, math.nan, math.inf):
        assert clip(g, None, 2, bad, at(3), None) == INVALID
    assert clip(g, None, 2, 1.0, None, None) == INVALID
    assert clip(g, None, 2, 1.0, ctypes.c_void_p(at(3).value + 4), None) == INVALID
    assert clip(None, None, 0, 1.0, at(3), None) == 0                    # nothing to do
    # outputs of another size, twice the same tensor, outputs over other entries
    assert clip(g, _list(b, (1 << 47, 8, 1, 0), ((1 << 47) + (1 << 40), 7, 0, 0)), 2, 1.0, at(3), None) == INVALID
    a = 1 << 45
    for entries in ([(a, 8, 1, 0), (a, 8, 1, 0)], [(a, 8, 1, 0), (a + 28, 8, 1, 0)], [(a + 28, 8, 0, 0), (a, 8, 1, 0)]):
        assert clip(_list(b, *entries), None, 2, 1.0, at(3), None) == INVALID
    two = _list(b, (a, 8, 1, 0), (a + 64, 8, 1, 0))
    for outs in ([(a, 8, 0, 0), (1 << 47, 8, 1, 0)],                     # its own memory in another type
                 [(a + 64, 8, 1, 0), (1 << 47, 8, 1, 0)], [(1 << 47, 8, 1, 0), (a + 60, 8, 1, 0)],
                 [(1 << 47, 8, 1, 0), ((1 << 47) + 30, 8, 0, 0)]):
        assert clip(two, _list(b, *outs), 2, 1.0, at(3), None) == INVALID


def test_binding_refuses_tensors(b):
    cpu = torch.zeros(4, 8)
    i32, f32 = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    with pytest.raises(ValueError, match="GPU"):
        b.bgpo_logits_logp(cpu, i32, f32)
    with pytest.raises(ValueError, match="matrix"):
        b.bgpo_logits_logp(f32, i32, f32)
    with pytest.raises(ValueError, match="GPU"):
        b.bgpo_logits_logp_bwd(cpu, i32, f32, None, f32, None, cpu)
    with pytest.raises(ValueError, match="GPU"):
        b.GradList([cpu])
    with pytest.raises(ValueError, match="GPU"):
        b.bgpo_policy_loss(b.PolicyLoss(4, 8), cpu, None, None, f32, cpu, None, f32, None)
    with pytest.raises(ValueError, match="GPU"):
        b.bgpo_preference_loss(b.PreferenceLoss(4, 8), cpu, cpu, None, None, None, None, None, None, None, None, None, f32, None)
