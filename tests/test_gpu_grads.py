"""Norm of a list of gradients and clipping vs float64 numpy.

The norm sums squares in float64: n terms agree within (n + 64) 2^-52 relative, the
root halves it.  Clipping multiplies by max / norm rounded to fp32 and rounds once
to the output's type: 2^-24 twice, and 2^-8 more for bf16.
"""
import math

import numpy as np
import pytest
import torch

from oracle import policy as oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def lib():
    from paper_2510_11683_amd import bgpo
    return bgpo


def _make(sizes, dtypes, seed=0, scale=1e-3, offset=1):
    """Tensors of the sizes, each `offset` elements off the last one's end in an
    array of its type (so that most are not aligned)."""
    rng = np.random.default_rng([seed, len(sizes)])
    out = []
    for t in (torch.float32, torch.bfloat16):
        at = [i for i in range(len(sizes)) if dtypes[i % len(dtypes)] == t]
        big = torch.full((sum(sizes[i] + offset for i in at) + offset,), 5.0, dtype=t, device="cuda")
        pos = offset
        for i in at:
            v = big[pos:pos + sizes[i]]
            v.copy_(torch.from_numpy((scale * rng.standard_normal(sizes[i])).astype(np.float32)))
            out.append((i, v))
            pos += sizes[i] + offset
    return [v for _, v in sorted(out, key=lambda p: p[0])]


def _norm(tensors, kind=0, flags=None):
    b = lib()
    n = torch.full((1,), 7.0, dtype=torch.float64, device="cuda")
    b.bgpo_grad_norm(b.GradList(tensors), n, b.grad_workspace(), kind, flags)
    return n


def _host(tensors):
    return [t.double().cpu().numpy() for t in tensors]


LISTS = [[], [0], [1], [3], [5, 0, 7], [16384], [16385, 1, 8191], [1 << 20], [100003, 64, 64, 4096, 12345],
         [37] * 300, [(i * 7919) % 5000 for i in range(900)], [5_000_001, 17]]


@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: f"{len(s)}x{max(s, default=0)}")
@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.bfloat16,), (torch.float32, torch.bfloat16)])
def test_norm_and_clip(sizes, dtypes):
    b = lib()
    g = _make(sizes, dtypes)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    n = _norm(g, flags=flags)
    h = _host(g)
    want = oracle.grad_norm(h)
    assert abs(float(n) - want) <= (sum(sizes) + 64) * 2.0 ** -52 * want
    assert float(_norm(g, b.BGPO_NORM_MAX)) == oracle.grad_norm(h, "max") and int(flags) == 0
    assert torch.equal(_norm(g), n)
    for max_norm in (0.3 * want, 2 * want + 1.0, 0.0):
        ref = oracle.grad_clip(h, max_norm, float(n))
        for out_t in (None, torch.float32, torch.bfloat16):
            src = [t.clone() for t in g]
            big = None if out_t is None else torch.full((sum(sizes) + len(sizes) + 1,), 3.0, dtype=out_t, device="cuda")
            out, pos = src, 1
            if big is not None:
                out = []
                for s in sizes:
                    out.append(big[pos:pos + s])
                    pos += s + 1
            b.bgpo_grad_clip(b.GradList(src), max_norm, n, None if big is None else b.GradList(out))
            for o, r, t, s in zip(out, ref, g, src):
                tol = 2 * 2.0 ** -24 + (2.0 ** -8 if o.dtype == torch.bfloat16 else 0.0)
                assert (np.abs(o.double().cpu().numpy() - r) <= tol * np.abs(r)).all()
                if max_norm > want:
                    assert torch.equal(o, t.to(o.dtype))
                if big is not None:
                    assert torch.equal(s, t)
            if big is not None:                       # what lies between the outputs is left alone
                keep = torch.ones(big.numel(), dtype=torch.bool)
                pos = 1
                for s in sizes:
                    keep[pos:pos + s] = False
                    pos += s + 1
                assert (big[keep.cuda()] == 3.0).all()


def test_values_at_the_limits():
    """Squares past fp32's range in either direction, NaN and infinities anywhere."""
    b = lib()
    for v in (3e38, 1e-38, 2.0 ** -133):
        g = [torch.full((1001,), v, device="cuda"), torch.full((77,), -v, device="cuda").bfloat16()]
        h = _host(g)
        want = oracle.grad_norm(h)
        n = _norm(g)
        assert abs(float(n) - want) <= 2000 * 2.0 ** -52 * want and float(_norm(g, 1)) == oracle.grad_norm(h, "max")
    for bad in (math.nan, math.inf, -math.inf):
        for where in (0, 500, 40000):
            g = _make([40001, 900], (torch.float32, torch.bfloat16))
            g[0][where] = bad
            before = [t.clone() for t in g]
            for kind in (0, 1):
                flags = torch.zeros(1, dtype=torch.int32, device="cuda")
                n = _norm(g, kind, flags)
                assert int(flags) == b.BGPO_FLAG_NONFINITE
                assert math.isnan(float(n)) if math.isnan(bad) else float(n) == math.inf
                out = [torch.empty_like(t) for t in g]
                b.bgpo_grad_clip(b.GradList(g), 1e-3, n, b.GradList(out))     # copies
                b.bgpo_grad_clip(b.GradList(g), 1e-3, n)                      # leaves alone
                for t, o, s in zip(g, out, before):
                    assert torch.equal(t.view(torch.int16), s.view(torch.int16)) and torch.equal(o[1:where], s[1:where])


def test_entry_that_is_its_own_output():
    b = lib()
    g = _make([1000, 333], (torch.float32,))
    h = _host(g)
    other = torch.empty(333, dtype=torch.bfloat16, device="cuda")
    n = _norm(g)
    b.bgpo_grad_clip(b.GradList(g), 1e-3, n, b.GradList([g[0], other]))
    want = oracle.grad_clip(h, 1e-3, float(n))
    assert np.allclose(g[0].double().cpu().numpy(), want[0], rtol=2 ** -23, atol=0)
    assert np.allclose(other.double().cpu().numpy(), want[1], rtol=2 ** -7.9, atol=0)
    assert np.array_equal(_host(g)[1], h[1])


def test_list_follows_its_tensors():
    """A list that was built once is looked up again after its tensors moved."""
    b = lib()
    p = torch.ones(4096, device="cuda")
    lst, ws = b.GradList([p]), b.grad_workspace()
    n = torch.empty(1, dtype=torch.float64, device="cuda")
    b.bgpo_grad_norm(lst, n, ws)
    assert float(n) == 64.0
    p.data = torch.full((4096,), 2.0, device="cuda")
    b.bgpo_grad_norm(lst, n, ws)
    assert float(n) == 128.0


def test_large_tensor():
    """Offsets past 2^32 bytes and 2^31 elements."""
    b = lib()
    n_el = (1 << 31) + 12345
    t = torch.zeros(n_el, dtype=torch.bfloat16, device="cuda")
    t[-1], t[0], t[1 << 31] = 3.0, 4.0, 12.0
    n = _norm([t])
    assert float(n) == 13.0
    b.bgpo_grad_clip(b.GradList([t]), 6.5, n)
    assert [float(t[i]) for i in (0, 1 << 31, n_el - 1)] == [2.0, 6.0, 1.5]


def test_deterministic_and_replays():
    b = lib()
    g = _make([(i * 7919) % 50000 + 1 for i in range(250)], (torch.float32, torch.bfloat16))
    out = [torch.empty(t.numel(), dtype=torch.bfloat16, device="cuda") for t in g]
    gl, ol, ws = b.GradList(g), b.GradList(out), b.grad_workspace()
    n = torch.empty(1, dtype=torch.float64, device="cuda")

    def step():
        b.bgpo_grad_norm(gl, n, ws)
        b.bgpo_grad_clip(gl, 0.1, n, ol)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        for t in g:
            t.mul_(1.5)
        got = []
        for run in (step, step, graph.replay):
            n.fill_(9.0)
            ws.fill_(170)
            for t in out:
                t.fill_(1.0)
            run()
            torch.cuda.synchronize()
            got.append([n.clone()] + [t.clone() for t in out])
        assert all(torch.equal(p, q) for o in got[1:] for p, q in zip(got[0], o))
