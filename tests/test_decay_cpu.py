"""Refusals of the entry points of decayed linear attention and beam search: before any device work, so without a GPU."""
import ctypes

import pytest
import torch

import paper_2603_04127_amd as dk

A, WS, BIG = 1 << 20, 1 << 24, 1 << 30   # aligned, never dereferenced: every call below fails in the checks or enqueues nothing


def _p(**kw):
    base = dict(B=1, H=1, L=64, dk=16, dv=8, io_dtype=dk.DARK_F32, layout=dk.BHLD, scale=0.0, sched_segments=0)
    base.update(kw)
    return ctypes.byref(dk.DecayParams(*base.values()))


BAD = [dict(H=0), dict(B=-1), dict(L=-1), dict(dk=0), dict(dv=0), dict(io_dtype=7), dict(layout=2), dict(scale=-1.0), dict(scale=float("nan")),
       dict(scale=float("inf")), dict(sched_segments=-1)]
TOO_LARGE = [dict(dk=257), dict(dv=300), dict(B=1 << 20, H=8), dict(L=(1 << 30) + 1)]


def test_forward_refusals():
    f = dk.lib().dark_decay_fwd
    ok = (A, A, A, A, None, None, A, None, None, 0, None)
    for kw in BAD:
        assert f(_p(**kw), *ok) == dk.DARK_EINVAL, kw
    for kw in TOO_LARGE:
        assert f(_p(**kw), *ok) == dk.DARK_EUNSUPPORTED, kw
    assert f(None, *ok) == dk.DARK_EINVAL
    for i in (0, 1, 2, 3, 6):
        assert f(_p(), *(None if j == i else x for j, x in enumerate(ok))) == dk.DARK_EINVAL, i
    for i, bad in ((0, A + 8), (3, A + 2), (4, A + 1), (5, A + 4), (6, A + 2), (7, A + 8)):
        assert f(_p(), *(bad if j == i else x for j, x in enumerate(ok))) == dk.DARK_EALIGN, i
    # states that overlap without being the same
    assert f(_p(), A, A, A, A, None, A, A, A + 256, None, 0, None) == dk.DARK_EINVAL
    # several segments need a workspace
    need = dk.lib().dark_decay_workspace_bytes(_p(L=1000, sched_segments=4), 0)
    assert need >= 4 * 16 * 8 * 4
    for ws, n, status in ((None, 0, dk.DARK_EWORKSPACE), (WS, need - 1, dk.DARK_EWORKSPACE), (WS + 16, need, dk.DARK_EALIGN)):
        assert f(_p(L=1000, sched_segments=4), A, A, A, A, None, None, A, None, ws, n, None) == status
    # nothing to do
    assert f(_p(B=0), *ok) == dk.DARK_OK
    assert f(_p(L=0), None, None, None, A, None, None, None, None, None, 0, None) == dk.DARK_OK
    assert f(_p(L=0), None, None, None, None, None, None, None, A, None, 0, None) == dk.DARK_EINVAL


def test_backward_refusals():
    f = dk.lib().dark_decay_bwd
    ok = (A, A, A, A, None, None, A, None, A, A, A, None, None, 0, None)
    for kw in BAD:
        assert f(_p(**kw), *ok) == dk.DARK_EINVAL, kw
    for i in (0, 1, 2, 3, 6):
        assert f(_p(), *(None if j == i else x for j, x in enumerate(ok))) == dk.DARK_EINVAL, i
    for i in (0, 1, 2, 6, 7, 8, 9, 10, 11):
        assert f(_p(), *(A + 8 if j == i else x for j, x in enumerate(ok))) == dk.DARK_EALIGN, i
    assert f(_p(), A, A, A, A, None, None, A, A, A, A, A, A, None, 0, None) == dk.DARK_EINVAL       # dS_in on dS_out
    assert f(_p(), A, A, A, A, None, A, A, None, A, A, A, A + 256, None, 0, None) == dk.DARK_EINVAL   # dS_in on S_in
    need = dk.lib().dark_decay_workspace_bytes(_p(L=1000, sched_segments=4), 1)
    assert need >= 2 * 4 * 16 * 8 * 4
    assert f(_p(L=1000, sched_segments=4), *ok[:-3], WS, need - 1, None) == dk.DARK_EWORKSPACE
    assert f(_p(B=0), *ok) == dk.DARK_OK


def test_step_refusals():
    f = dk.lib().dark_decay_step
    far = A + (1 << 22)
    ok = (A, A, A, A, None, 1, A, A, far, None)
    for kw in BAD:
        assert f(_p(**kw), *ok) == dk.DARK_EINVAL, kw
    for i in (0, 1, 2, 3, 6, 7, 8):
        assert f(_p(), *(None if j == i else x for j, x in enumerate(ok))) == dk.DARK_EINVAL, i
    for i in (0, 1, 2, 8):   # aligned as their elements are
        assert f(_p(), *(A + 2 if j == i else x for j, x in enumerate(ok))) == dk.DARK_EALIGN, i
        assert f(_p(io_dtype=dk.DARK_BF16), *(A + 1 if j == i else x for j, x in enumerate(ok))) == dk.DARK_EALIGN, i
    for i in (6, 7):
        assert f(_p(), *(A + 8 if j == i else x for j, x in enumerate(ok))) == dk.DARK_EALIGN, i
    assert f(_p(), A, A, A, A, None, 2, A, A, far, None) == dk.DARK_EINVAL          # without parents the rows are the batch's
    assert f(_p(), A, A, A, A, A, 0, A, far, far, None) == dk.DARK_EINVAL
    assert f(_p(), A, A, A, A, A, 1, A, A, far, None) == dk.DARK_EINVAL             # a step through parents is not in place
    assert f(_p(B=2), A, A, A, A, A, 3, A, A + 2 * 16 * 8 * 4, far, None) == dk.DARK_EINVAL
    assert f(_p(B=2), A, A, A, A, None, 2, A, A + 16 * 8 * 4, far, None) == dk.DARK_EINVAL
    assert f(_p(B=0), A, A, A, A, None, 0, A, A, far, None) == dk.DARK_OK


def _b(**kw):
    base = dict(B=1, n=4, V=100, io_dtype=dk.DARK_F32, eos=0, keep_slots=0)
    base.update(kw)
    return ctypes.byref(dk.BeamParams(*base.values()))


def test_selection_refusals():
    f = dk.lib().dark_beam_select
    ok = (A, A, None, A, A, A, WS, BIG, None)
    for kw in (dict(B=-1), dict(n=0), dict(V=0), dict(io_dtype=3)):
        assert f(_b(**kw), *ok) == dk.DARK_EINVAL, kw
    for kw in (dict(n=33), dict(n=32, V=1 << 26), dict(B=65536, n=1), dict(n=32, V=3_000_000)):
        assert f(_b(**kw), *ok) == dk.DARK_EUNSUPPORTED, kw
    for i in (0, 1, 3, 4, 5):
        assert f(_b(), *(None if j == i else x for j, x in enumerate(ok))) == dk.DARK_EINVAL, i
    for eos in (-1, 100):
        assert f(_b(eos=eos), A, A, A, A, A, A, WS, BIG, None) == dk.DARK_EINVAL
    assert f(_b(), A + 4, *ok[1:]) == dk.DARK_EALIGN
    need = dk.lib().dark_beam_workspace_bytes(_b())
    assert need > 0 and f(_b(), *ok[:6], WS, need - 1, None) == dk.DARK_EWORKSPACE
    assert f(_b(), *ok[:6], WS + 8, need, None) == dk.DARK_EALIGN
    assert f(_b(B=0), None, None, None, None, None, None, None, 0, None) == dk.DARK_OK


def test_reorder_refusals():
    f = dk.lib().dark_state_reorder
    ptrs, sizes = (ctypes.c_void_p * 2)(A, A + 4096), (ctypes.c_size_t * 2)(64, 64)
    assert f(-1, 4, A, 2, ptrs, sizes, None) == dk.DARK_EINVAL
    assert f(1, 0, A, 2, ptrs, sizes, None) == dk.DARK_EINVAL
    assert f(1, 4, A, -1, ptrs, sizes, None) == dk.DARK_EINVAL
    assert f(1, 33, A, 2, ptrs, sizes, None) == dk.DARK_EUNSUPPORTED
    assert f(65536, 4, A, 2, ptrs, sizes, None) == dk.DARK_EUNSUPPORTED
    assert f(1, 4, None, 2, ptrs, sizes, None) == dk.DARK_EINVAL
    assert f(1, 4, A + 2, 2, ptrs, sizes, None) == dk.DARK_EALIGN
    ptrs[1] = A + 4
    assert f(1, 4, A, 2, ptrs, sizes, None) == dk.DARK_EALIGN
    ptrs[1] = None
    assert f(1, 4, A, 2, ptrs, sizes, None) == dk.DARK_EINVAL
    assert f(0, 4, A, 2, ptrs, sizes, None) == dk.DARK_OK and f(1, 4, A, 0, None, None, None) == dk.DARK_OK


def test_reorder_refuses_before_anything_has_moved():
    # a row too long for a launch, behind more tensors than one launch takes: without a GPU a launch would be DARK_EHIP
    f = dk.lib().dark_state_reorder
    for unit in (1, 4, 16):
        for where in (0, 1, 16, 39):
            sizes = (ctypes.c_size_t * 40)(*([64] * 40))
            sizes[where] = unit * ((1 << 31) + 1)
            ptrs = (ctypes.c_void_p * 40)(*(A + 4096 * i if i != where else 1 << 40 for i in range(40)))
            assert f(1, 4, A - 4096, 40, ptrs, sizes, None) == dk.DARK_EUNSUPPORTED, (unit, where)
    assert f(1, 4, A - 4096, 1, (ctypes.c_void_p * 1)(1 << 40), (ctypes.c_size_t * 1)((1 << 64) - 16), None) == dk.DARK_EUNSUPPORTED


def test_results_lie_on_nothing_else():
    far = [A + (i << 20) for i in range(16)]   # every argument a place of its own, then one result on another argument
    fwd, bwd, step, select, reorder = (getattr(dk.lib(), "dark_" + name) for name in ("decay_fwd", "decay_bwd", "decay_step", "beam_select", "state_reorder"))
    args = far[:6] + far[6:8] + [None, 0, None]   # Q, K, V, log_decay, lengths, S_in; out, S_out
    for result, other in [(6, j) for j in range(6)] + [(7, j) for j in (0, 1, 2, 3, 4, 6)]:
        assert fwd(_p(), *(far[other] if i == result else x for i, x in enumerate(args))) == dk.DARK_EINVAL, (result, other)
    assert fwd(_p(), *(far[2] + 64 * 8 * 4 - 16 if i == 6 else x for i, x in enumerate(args))) == dk.DARK_EINVAL   # out begins in V's last row
    args = far[:12] + [None, 0, None]   # Q, K, V, log_decay, lengths, S_in, dOut, dS_out; dQ, dK, dV, dS_in
    for result in range(8, 12):
        for other in range(result):
            assert bwd(_p(), *(far[other] if i == result else x for i, x in enumerate(args))) == dk.DARK_EINVAL, (result, other)
    args = far[:5] + [1] + far[6:9] + [None]   # q, k, v, log_decay, parent, rows, S_in; S_out, out
    for result, other in [(7, j) for j in (0, 1, 2, 3, 4, 6)] + [(8, j) for j in (0, 1, 2, 3, 4, 6, 7)]:
        assert step(_p(), *(far[other] if i == result else x for i, x in enumerate(args))) == dk.DARK_EINVAL, (result, other)
    args = far[:6] + [WS, BIG, None]   # logits, scores, finished; scores, parents, tokens
    for result, other in ((3, 0), (3, 2), (4, 0), (4, 1), (4, 2), (4, 3), (5, 0), (5, 1), (5, 2), (5, 3), (5, 4)):
        assert select(_b(), *(far[other] if i == result else x for i, x in enumerate(args))) == dk.DARK_EINVAL, (result, other)
    assert select(_b(), far[0], far[1], None, far[1] + 4, far[4], far[5], WS, BIG, None) == dk.DARK_EINVAL   # scores, shifted
    sizes = (ctypes.c_size_t * 3)(64, 64, 64)
    for places in ((A, A, far[1]), (A, far[1], A + 3 * 64), (far[1], far[2], far[3] - 16)):   # twice the same, the last row, the parents
        assert reorder(1, 4, far[3], 3, (ctypes.c_void_p * 3)(*places), sizes, None) == dk.DARK_EINVAL


def test_binding_refusals():
    x, a = torch.zeros(2, 3, 10, 16), torch.zeros(3)
    with pytest.raises(ValueError, match="layout"):
        dk.dark_decay_fwd(x, x, x, a, layout="bldh")
    with pytest.raises(ValueError, match="log_decay"):
        dk.dark_decay_fwd(x, x, x, torch.zeros(10))
    with pytest.raises(ValueError, match="log_decay"):
        dk.dark_decay_fwd(x, x, x, a.double())
    with pytest.raises(ValueError, match="lengths"):
        dk.dark_decay_fwd(x, x, x, a, lengths=torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="state"):
        dk.dark_decay_fwd(x, x, x, a, state=torch.zeros(2, 3, 16, 8))
    with pytest.raises(ValueError, match="same"):
        dk.dark_decay_fwd(x, x[:, :, :9], x, a)
    with pytest.raises(TypeError):
        dk.dark_decay_fwd(x, x, x.bfloat16(), a)
    with pytest.raises(TypeError):
        dk.dark_decay_fwd(x.half(), x.half(), x.half(), a)
    with pytest.raises(ValueError, match="GPU"):
        dk.dark_decay_fwd(x, x, x, a)
    with pytest.raises(ValueError, match="dOut"):
        dk.dark_decay_bwd(x, x, x, a, x.bfloat16())
    with pytest.raises(ValueError, match="unknown"):
        dk.dark_decay_bwd(x, x, x, a, x, need=("dW",))
    q = x[:, :, 0]
    with pytest.raises(ValueError, match="state_out"):
        dk.dark_decay_step(q, q, q, a, torch.zeros(2, 3, 16, 16), parent=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="state"):
        dk.dark_decay_step(q, q, q, a, torch.zeros(3, 3, 16, 16))
    with pytest.raises(ValueError, match="parent"):
        dk.dark_decay_step(q, q, q, a, torch.zeros(2, 3, 16, 16), parent=torch.zeros(3, dtype=torch.int32), state_out=torch.zeros(2, 3, 16, 16))
    logits, scores = torch.zeros(2, 4, 50), torch.zeros(2, 4)
    with pytest.raises(ValueError, match="scores"):
        dk.dark_beam_select(logits, scores.double())
    with pytest.raises(ValueError, match="finished"):
        dk.dark_beam_select(logits, scores, finished=scores)
    with pytest.raises(ValueError, match="GPU"):
        dk.dark_beam_select(logits, scores)
    with pytest.raises(ValueError, match="parent"):
        dk.dark_state_reorder([logits], torch.zeros(2, 4))
    with pytest.raises(ValueError):
        dk.dark_state_reorder([torch.zeros(7, 3)], torch.zeros(2, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        dk.dark_state_reorder([logits], torch.zeros(2, 4, dtype=torch.int32))


def test_workspaces_follow_the_call():
    need = lambda **kw: dk.lib().dark_decay_workspace_bytes(_p(**kw), 0)
    assert need() == 0 and need(L=0) == 0 and need(B=0, L=5000) == 0 and need(dk=0) == 0
    assert need(L=5000) > 0 and need(L=5000, B=64, H=16) == 0       # enough heads: nothing is cut
    assert dk.lib().dark_decay_workspace_bytes(_p(L=5000), 1) > 0
    w = lambda **kw: dk.lib().dark_beam_workspace_bytes(_b(**kw))
    assert 0 < w() < w(V=100000) and w(B=0) == 0 and w(n=0) == 0
