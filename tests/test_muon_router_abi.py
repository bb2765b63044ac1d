"""What the Muon and router entry points refuse, and their workspace sizes: host code only, no GPU needed.  Addresses are made up; a
call that refuses looks at none of them."""
import ctypes

import numpy as np
import pytest

from paper_2601_02609_amd import binding as B
from paper_2601_02609_amd import build

AT = 1 << 20                                             # an address with every alignment
ABC = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def L():
    if not build.is_built():
        build.build(verbose=False)
    return B.lib()


def _table(*entries):
    t = np.zeros(len(entries), dtype=np.dtype(B._Matrix))
    for i, e in enumerate(entries):
        for k, v in dict(param=AT, out_bf16=AT, grad=AT, momentum=AT, rows=4, cols=6, lr_scale=1.0).items():
            t[i][k] = v
        for k, v in e.items():
            t[i][k] = v
    return t


def _bytes(L, *entries):
    t = _table(*entries)
    return L.cce_muon_workspace_bytes(t.ctypes.data, len(t))


def test_workspace_bytes(L):
    assert _bytes(L, {}) == 256                          # few rows: a workgroup alone, no workspace
    assert _bytes(L, dict(rows=0, cols=1 << 40)) == 256 and _bytes(L, dict(rows=128, cols=448)) == 256
    one = _bytes(L, dict(rows=512, cols=640))
    assert one >= 512 * 640 * 5 + 512 * 512 * 4 and one <= 1.1 * (512 * 640 * 5 + 512 * 512 * 4)
    assert _bytes(L, *[dict(rows=640, cols=512)] * 3) == 3 * one
    large = _bytes(L, dict(rows=4096, cols=2048))
    assert 0 < large - (4096 * 2048 * 5 + 2048 * 2048 * 4) < (64 << 20) + (1 << 20)
    assert _bytes(L, *[dict(rows=4096, cols=4096)] * 300) <= 3 << 30
    assert _bytes(L, dict(rows=1 << 14, cols=1 << 16)) > 0
    for sizes in ((1 << 24, 65), (1 << 30, 1), (16385, 16385), (1 << 40, 1 << 40)):
        assert _bytes(L, dict(rows=sizes[0], cols=sizes[1])) == 0
    assert _bytes(L, dict(rows=-1)) == 0 and L.cce_muon_workspace_bytes(None, 1) == 0
    t = _table({})
    assert L.cce_muon_workspace_bytes(t.ctypes.data, 0) == 0


def _orthogonalize(L, entries, coefficients=ABC, steps=5, eps=1e-7, workspace=AT, size=1 << 30, count=None):
    t = _table(*entries)
    c = None if coefficients is None else np.ascontiguousarray(np.broadcast_to(np.asarray(coefficients, dtype=np.float32), (max(steps, 1), 3)))
    return L.cce_orthogonalize_multi(t.ctypes.data, len(t) if count is None else count, None if c is None else c.ctypes.data, steps, eps, workspace, size, None)


def test_orthogonalize_refusals(L):
    bad = [dict(grad=0), dict(grad=AT + 2), dict(out_bf16=0), dict(out_bf16=AT + 1), dict(rows=-1), dict(grad_bf16=2), dict(reserved=1)]
    for e in bad:
        assert _orthogonalize(L, [{}, e]) == B.CCE_ERR_INVALID, e
    assert _orthogonalize(L, [{}], count=0) == B.CCE_ERR_INVALID
    assert _orthogonalize(L, [dict(rows=1 << 16, cols=1 << 16)]) == B.CCE_ERR_UNSUPPORTED
    for kw in (dict(steps=0), dict(steps=17), dict(eps=-1.0), dict(eps=float("nan")), dict(coefficients=None), dict(workspace=None), dict(workspace=AT + 128),
               dict(size=255), dict(coefficients=(float("inf"), 0.0, 0.0))):
        assert _orthogonalize(L, [{}], **kw) == B.CCE_ERR_INVALID, kw
    assert _orthogonalize(L, [dict(rows=512, cols=640)], size=1 << 20) == B.CCE_ERR_INVALID
    # 2 x + x^3 + x^5 takes 1 to 4; 3 x - 61 x^3 leaves the operands' range; 1.6 x grows to 1.6^2 = 2.56 in the second step
    for c, steps in (((2.0, 1.0, 1.0), 1), ((3.0, -61.0, 0.0), 1), ((1.6, 0.0, 0.0), 2)):
        assert _orthogonalize(L, [{}], coefficients=c, steps=steps) == B.CCE_ERR_UNSUPPORTED, c


def test_bound_on_singular_values_is_the_polynomials_largest_value():
    """What the refusal goes by, against a fine grid, for the coefficients that the header allows or not."""
    L = B.lib()
    rng = np.random.default_rng(0)
    refused = 0
    for _ in range(300):
        a, b, c = (float(np.float32(v)) for v in (rng.uniform(0.5, 6.0), rng.uniform(-12.0, 4.0), rng.uniform(-3.0, 8.0)))
        x = np.linspace(0.0, 1.0, 20001)
        top = np.abs(a * x + b * x ** 3 + c * x ** 5).max()
        if abs(top - 2.5) < 1e-3:
            continue
        # an allowed call goes on to the workspace's size, which is too small
        rc = _orthogonalize(L, [{}], coefficients=(a, b, c), steps=1, size=255)
        assert rc == B.CCE_ERR_INVALID
        got = _orthogonalize(L, [dict(rows=0)], coefficients=(a, b, c), steps=1)
        assert (got == B.CCE_ERR_UNSUPPORTED) == (top > 2.5), (a, b, c, top, got)
        refused += top > 2.5
    assert 30 < refused < 270


def test_muon_step_refusals(L):
    def step(entries, lr=0.1, mu=0.9, clip=None):
        t = _table(*entries)
        c = np.ascontiguousarray(np.broadcast_to(np.asarray(ABC, dtype=np.float32), (5, 3)))
        return L.cce_muon_multi_step(t.ctypes.data, len(t), lr, mu, 1, c.ctypes.data, 5, 1e-7, clip, AT, 1 << 30, None)

    for e in (dict(param=0), dict(param=AT + 2), dict(momentum=0), dict(momentum=AT + 1), dict(out_bf16=AT + 1), dict(lr_scale=-1.0), dict(weight_decay=float("nan"))):
        assert step([e]) == B.CCE_ERR_INVALID, e
    for kw in (dict(lr=-0.1), dict(lr=float("nan")), dict(mu=1.0), dict(mu=-0.1), dict(clip=AT + 2)):
        assert step([{}], **kw) == B.CCE_ERR_INVALID, kw


def test_nothing_to_do_is_done(L):
    """Matrices without values alone: accepted, and nothing is launched."""
    assert _orthogonalize(L, [dict(rows=0, grad=0, out_bf16=0), dict(cols=0, grad=0, out_bf16=0)]) in (B.CCE_OK, B.CCE_ERR_HIP)


def _forward(L, **kw):
    a = dict(logits=AT, bf16=0, labels=None, N=10, E=8, k=2, renormalize=1, ignore=-100, indices=AT, weights=AT, lse=AT, counts=AT, sums=AT, losses=AT, workspace=AT, size=1 << 20)
    a.update(kw)
    return L.cce_router_forward(*a.values(), None)


def _backward(L, **kw):
    a = dict(logits=AT, bf16=0, indices=AT, lse=AT, counts=AT, d_weights=None, d_losses=None, N=10, E=8, k=2, renormalize=1, d_logits=AT)
    a.update(kw)
    return L.cce_router_backward(*a.values(), None)


def test_router_refusals(L):
    common = [dict(N=0), dict(N=-1), dict(E=0), dict(k=0), dict(k=9), dict(bf16=2), dict(renormalize=2), dict(logits=None), dict(logits=AT + 2), dict(indices=None),
              dict(indices=AT + 2), dict(lse=None), dict(lse=AT + 1), dict(counts=None)]
    for e in common + [dict(weights=None), dict(sums=None), dict(losses=None), dict(workspace=None), dict(workspace=AT + 4), dict(size=8), dict(labels=AT + 2), dict(losses=AT + 2)]:
        assert _forward(L, **e) == B.CCE_ERR_INVALID, e
    for e in common + [dict(d_logits=None), dict(d_logits=AT + 2), dict(d_weights=AT + 2), dict(d_losses=AT + 1), dict(bf16=1, logits=AT + 1)]:
        assert _backward(L, **e) == B.CCE_ERR_INVALID, e
    for call in (_forward, _backward):
        for e in (dict(E=1025), dict(E=64, k=33), dict(N=1 << 31)):
            assert call(L, **e) == B.CCE_ERR_UNSUPPORTED, e


def test_router_workspace_bytes(L):
    ask = [L.cce_router_workspace_bytes(n, 64) for n in (1, 100, 1000, 10 ** 4, 10 ** 6, (1 << 31) - 1)]
    assert ask == sorted(ask) and ask[0] == 768 and ask[-1] == ask[-2] < 256 * (64 * 8 + 16)
    assert L.cce_router_workspace_bytes(0, 64) == 0 and L.cce_router_workspace_bytes(10, 1025) == 0 and L.cce_router_workspace_bytes(1 << 31, 8) == 0


def test_struct_is_the_headers(L):
    assert ctypes.sizeof(B._Matrix) == 64 and B._MATRIX.size == 64
    assert [name for name, _ in B._Matrix._fields_] == ["param", "out_bf16", "grad", "momentum", "rows", "cols", "lr_scale", "weight_decay", "grad_bf16", "reserved"]
