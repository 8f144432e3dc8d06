"""Refusals of the entry points of the gated delta rule: before any device work, so without a GPU."""
import ctypes

import pytest
import torch

import paper_2603_04127_amd as dk

A, WS, BIG = 1 << 20, 1 << 34, 1 << 30   # aligned, never dereferenced: every call below fails in the checks or enqueues nothing


def _p(**kw):
    base = dict(B=1, H=1, L=64, dk=16, dv=8, io_dtype=dk.DARK_F32, layout=dk.BHLD, scale=0.0)
    base.update(kw)
    return ctypes.byref(dk.DeltaParams(*base.values()))


BAD = [dict(H=0), dict(B=-1), dict(L=-1), dict(dk=0), dict(dv=0), dict(io_dtype=7), dict(layout=2), dict(scale=-1.0), dict(scale=float("nan")),
       dict(scale=float("inf"))]
TOO_LARGE = [dict(dk=257), dict(dv=300), dict(B=1 << 20, H=8), dict(L=(1 << 28) + 1), dict(B=1 << 10, L=(1 << 18) + 1), dict(layout=dk.BLHD, H=1 << 19)]


def _with(args, i, x):
    return tuple(x if j == i else y for j, y in enumerate(args))


def test_forward_refusals():
    f = dk.lib().dark_delta_fwd
    far = [A + (i << 20) for i in range(9)]   # Q, K, V, log_gate, beta, lengths, S_in; out, S_out
    ok = (*far[:5], None, None, far[7], None, WS, BIG, None)
    for kw in BAD:
        assert f(_p(**kw), *ok) == dk.DARK_EINVAL, kw
    for kw in TOO_LARGE:
        assert f(_p(**kw), *ok) == dk.DARK_EUNSUPPORTED, kw
    assert f(None, *ok) == dk.DARK_EINVAL
    for i in (0, 1, 2, 4, 7):
        assert f(_p(), *_with(ok, i, None)) == dk.DARK_EINVAL, i
    for i, bad in ((0, A + 8), (3, A + 2), (4, A + 1), (5, A + 2), (6, A + 4), (7, A + 2), (8, A + 8)):
        assert f(_p(), *_with(ok, i, bad)) == dk.DARK_EALIGN, i
    assert f(_p(), *far[:5], None, A, far[7], A + 256, WS, BIG, None) == dk.DARK_EINVAL   # states that overlap without being the same
    need = dk.lib().dark_delta_workspace_bytes(_p(), 0)
    assert need > 0
    for ws, n, status in ((None, BIG, dk.DARK_EWORKSPACE), (WS, need - 1, dk.DARK_EWORKSPACE), (WS + 16, need, dk.DARK_EALIGN)):
        assert f(_p(), *ok[:9], ws, n, None) == status
    assert f(_p(B=0), *ok) == dk.DARK_OK
    assert f(_p(L=0), *(None,) * 9, None, 0, None) == dk.DARK_OK
    args = (*far, WS, BIG, None)
    for result, other in [(7, j) for j in range(7)] + [(8, j) for j in (0, 1, 2, 3, 4, 5, 7)]:
        assert f(_p(), *_with(args, result, far[other])) == dk.DARK_EINVAL, (result, other)


def test_backward_refusals():
    f = dk.lib().dark_delta_bwd
    far = [A + (i << 20) for i in range(15)]   # Q, K, V, log_gate, beta, lengths, S_in, dOut, dS_out; dQ, dK, dV, dlog_gate, dbeta, dS_in
    ok = (*far, WS, BIG, None)
    for kw in BAD:
        assert f(_p(**kw), *ok) == dk.DARK_EINVAL, kw
    for kw in TOO_LARGE:
        assert f(_p(**kw), *ok) == dk.DARK_EUNSUPPORTED, kw
    for i in (0, 1, 2, 4, 7):
        assert f(_p(), *_with(ok, i, None)) == dk.DARK_EINVAL, i
    for i in range(15):
        assert f(_p(), *_with(ok, i, far[i] + 2)) == dk.DARK_EALIGN, i
    for result in range(9, 15):
        for other in range(result):
            assert f(_p(), *_with(ok, result, far[other])) == dk.DARK_EINVAL, (result, other)
    need = dk.lib().dark_delta_workspace_bytes(_p(), 1)
    assert need > dk.lib().dark_delta_workspace_bytes(_p(), 0) and f(_p(), *far, WS, need - 1, None) == dk.DARK_EWORKSPACE
    assert f(_p(B=0), *ok) == dk.DARK_OK
    assert f(_p(), *far[:9], None, None, None, None, None, None, WS, BIG, None) == dk.DARK_OK   # nothing is asked for


def test_step_refusals():
    f = dk.lib().dark_delta_step
    far = [A + (i << 20) for i in range(10)]   # q, k, v, log_gate, beta, parent, rows, S_in; S_out, out
    ok = (*far[:5], None, 1, *far[7:], None)
    for kw in BAD:
        if "L" not in kw:
            assert f(_p(**kw), *ok) == dk.DARK_EINVAL, kw
    assert f(_p(dk=257), *ok) == dk.DARK_EUNSUPPORTED and f(None, *ok) == dk.DARK_EINVAL
    for i in (0, 1, 2, 4, 7, 8, 9):
        assert f(_p(), *_with(ok, i, None)) == dk.DARK_EINVAL, i
    for i in (0, 1, 2, 3, 4, 9):   # aligned as their elements are
        assert f(_p(), *_with(ok, i, far[i] + 2)) == dk.DARK_EALIGN, i
    for i in (0, 1, 2, 9):
        assert f(_p(io_dtype=dk.DARK_BF16), *_with(ok, i, far[i] + 1)) == dk.DARK_EALIGN, i
    for i in (7, 8):
        assert f(_p(), *_with(ok, i, far[i] + 8)) == dk.DARK_EALIGN, i
    assert f(_p(), *_with(ok, 6, 2)) == dk.DARK_EINVAL                      # without parents the rows are the batch's
    args = (*far[:6], 1, *far[7:], None)
    assert f(_p(), *_with(args, 6, 0)) == dk.DARK_EINVAL
    for result, other in [(8, j) for j in (0, 1, 2, 3, 4, 5, 7)] + [(9, j) for j in (0, 1, 2, 3, 4, 5, 7, 8)]:
        assert f(_p(), *_with(args, result, far[other])) == dk.DARK_EINVAL, (result, other)
    assert f(_p(B=0), *_with(ok, 6, 0)) == dk.DARK_OK


def test_binding_refusals():
    x, a = torch.zeros(2, 3, 10, 16), torch.zeros(2, 3, 10)
    with pytest.raises(ValueError, match="layout"):
        dk.dark_delta_fwd(x, x, x, a, a, layout="bldh")
    with pytest.raises(ValueError, match="log_gate"):
        dk.dark_delta_fwd(x, x, x, torch.zeros(3), a)
    with pytest.raises(ValueError, match="log_gate"):
        dk.dark_delta_fwd(x, x, x, a.transpose(1, 2), a)
    with pytest.raises(ValueError, match="beta"):
        dk.dark_delta_fwd(x, x, x, None, a.bfloat16())
    with pytest.raises(ValueError, match="lengths"):
        dk.dark_delta_fwd(x, x, x, a, a, lengths=torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="state"):
        dk.dark_delta_fwd(x, x, x, a, a, state=torch.zeros(2, 3, 16, 8))
    with pytest.raises(ValueError, match="same"):
        dk.dark_delta_fwd(x, x[:, :, :9], x, a, a)
    with pytest.raises(TypeError):
        dk.dark_delta_fwd(x, x, x.bfloat16(), a, a)
    with pytest.raises(TypeError):
        dk.dark_delta_fwd(x.half(), x.half(), x.half(), a, a)
    with pytest.raises(ValueError, match="GPU"):
        dk.dark_delta_fwd(x, x, x, a, a)
    with pytest.raises(ValueError, match="dOut"):
        dk.dark_delta_bwd(x, x, x, a, a, x.bfloat16())
    with pytest.raises(ValueError, match="unknown"):
        dk.dark_delta_bwd(x, x, x, a, a, x, need=("dW",))
    with pytest.raises(ValueError, match="dbeta"):
        dk.dark_delta_bwd(x, x, x, a, a, x, grads={"dbeta": torch.zeros(2, 3)})
    q, b = x[:, :, 0], a[:, :, 0]
    with pytest.raises(ValueError, match="state_out"):
        dk.dark_delta_step(q, q, q, b, b, torch.zeros(2, 3, 16, 16), parent=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="state"):
        dk.dark_delta_step(q, q, q, b, b, torch.zeros(3, 3, 16, 16))
    with pytest.raises(ValueError, match="beta"):
        dk.dark_delta_step(q, q, q, b, torch.zeros(3), torch.zeros(2, 3, 16, 16))
