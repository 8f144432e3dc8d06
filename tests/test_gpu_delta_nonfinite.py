"""What elements that are not finite make of the results of the gated delta rule: the rows, columns and tensors that the header names, in every form of the kernels."""
import pytest
import torch

import paper_2603_04127_amd as dk
from tests import delta_util as U

pytestmark = pytest.mark.gpu
ARGS = ("Q", "K", "V", "a", "beta")
L = 300


def _device(p):
    return {k: None if t is None or k == "dtype" else t.cuda() for k, t in p.items()}


def _all(d):
    out, last = dk.dark_delta_fwd(*(d[k] for k in ARGS), state=d["state"], want_state=True)
    return {"out": out, "last": last, **dk.dark_delta_bwd(*(d[k] for k in ARGS), d["dOut"], state=d["state"], dstate=d["dstate"])}


def _spoilt(t, r, c):
    """For each result rows that are not finite at all, or columns of them ([:] before them all rows)."""
    after, upto = slice(r, None), slice(None, r + 1)
    forward = {"dQ": (after,), "dK": (after,), "dbeta": (after,), "dlog_gate": (slice(r + 1, None),)}
    backward = {"dK": (upto,), "dV": (upto,), "dbeta": (upto,), "dlog_gate": (upto,), "dstate": (slice(None),)}
    if t == "Q":
        return backward
    if t == "dOut":
        return {**backward, "dV": (upto, c), "dstate": (slice(None), c), "dQ": (slice(r, r + 1),)}
    if t == "V":
        return {**forward, "out": (after, c), "last": (slice(None), c)}
    both = {"out": (after,), "last": (slice(None),), "dQ": (after,), "dV": (upto,), **{k: (slice(None),) for k in ("dK", "dbeta", "dlog_gate", "dstate")}}
    return both


def _touched(t):
    """For each result whether rows behind (before) the element's chunk may differ from those without it."""
    before = {"dK", "dV", "dbeta", "dlog_gate", "dstate"}
    behind = {"dQ", "dK", "dbeta", "dlog_gate", "out", "last"}
    return (set() if t in ("Q", "dOut") else behind), (set() if t == "V" else before)


FORMS = [("bf16", 1, 64, 64), ("bf16", 3, 128, 128), ("bf16", 2, 33, 65), ("bf16", 70, 96, 80), ("bf16", 2, 256, 64), ("f32", 2, 64, 64), ("f32", 2, 31, 33), ("f32", 70, 64, 64),
         ("f32", 2, 256, 72)]


@pytest.mark.parametrize("r", [0, 130, 192, 255, L - 1])
@pytest.mark.parametrize("dtype,H,wide,high", FORMS)
def test_rows_and_columns_that_an_element_spoils(dtype, H, wide, high, r):
    C = 64 if dtype == "bf16" else 32
    p = U.problem(r + wide, 1, H, L, wide, high, dtype, state=True, dstate=True)
    p["a"][:, :, 210] = float("-inf")   # a gate that keeps nothing stops no NaN
    d = _device(p)
    clean = _all(d)
    assert all(torch.isfinite(t).all() for t in clean.values())
    h, c = H - 1, min(7, high - 1)
    first, end = r // C * C, (r // C + 1) * C
    for name in ("Q", "K", "V", "a", "beta", "dOut"):
        for bad in (float("nan"), float("inf")):
            e = {**d, name: d[name].clone()}
            wide_at = (0, h, r) if name in ("a", "beta") else (0, h, r, c if name in ("V", "dOut") else min(3, wide - 1))
            e[name][wide_at] = bad
            got = _all(e)
            want = _spoilt(name, r, c)
            behind, before = _touched(name)
            for k, t in got.items():
                where = (name, bad, k)
                assert torch.equal(t[0, :h], clean[k][0, :h]), where            # other heads
                x, y = t[0, h], clean[k][0, h]
                if k in want:
                    part = x[want[k][0]] if len(want[k]) == 1 else x[want[k][0], want[k][1]]
                    bad_rows = ~torch.isfinite(part)
                    if name == "beta" and k == "dbeta":
                        bad_rows[r] = True                                      # a beta's own row
                    assert bad_rows.all(), where
                if k in ("last", "dstate"):
                    if k not in behind | before:
                        assert torch.equal(x, y), where
                    continue
                if k == "out" and name == "Q" or k == "dQ" and name == "dOut":
                    assert torch.equal(torch.cat([x[:first], x[end:]]), torch.cat([y[:first], y[end:]])), where
                    continue
                if k not in behind:
                    assert torch.equal(x[end:], y[end:]), where
                if k not in before:
                    assert torch.equal(x[:first], y[:first]), where
