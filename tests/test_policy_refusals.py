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
    for h in ("bgpo_policy.h",):
        src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", h)).read(), flags=re.S)
        names |= set(re.findall(r"\b(bgpo_\w+)\s*\(", src))
    assert {"bgpo_logits_logp", "bgpo_logits_logp_bwd"} <= names
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
              (dict(scale=-1.0), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID),
              (dict(reserved=1), INVALID), (dict(rows=1 << 31), UNSUPPORTED),
              (dict(V=(1 << 24) + 1, ld=1 << 25), UNSUPPORTED), (dict(ld=(1 << 40) + 1), INVALID)]


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


def test_binding_refuses_tensors(b):
    cpu = torch.zeros(4, 8)
    i32, f32 = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    with pytest.raises(ValueError, match="GPU"):
        b.bgpo_logits_logp(cpu, i32, f32)
    with pytest.raises(ValueError, match="matrix"):
        b.bgpo_logits_logp(f32, i32, f32)
    with pytest.raises(ValueError, match="GPU"):
        b.bgpo_logits_logp_bwd(cpu, i32, f32, None, f32, None, cpu)
