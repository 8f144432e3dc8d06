"""The gated delta rule's results against the fp64 oracle within close bounds (delta_terms.py), in every form of the kernels."""
import pytest
import torch

import paper_2603_04127_amd as dk
from tests import delta_terms as T, delta_util as U

pytestmark = pytest.mark.gpu


def _run(p, aligned=False, layout="bhld"):
    turn = (lambda t: t) if layout == "bhld" else (lambda t: t.transpose(1, 2).contiguous())
    d = {k: turn(p[k]).cuda() for k in T.U_NAMES}
    n, s, ds = (None if p[k] is None else p[k].cuda() for k in ("lengths", "state", "dstate"))
    x = [d[k] for k in ("Q", "K", "V", "a", "beta")]
    out, last = dk.dark_delta_fwd(*x, lengths=n, state=s, want_state=True, layout=layout)
    got = {"out": out, "last": last, **dk.dark_delta_bwd(*x, d["dOut"], lengths=n, state=s, dstate=ds, layout=layout)}
    want, _ = U.oracle(p)
    size = T.sizes_of(p, aligned=aligned)
    for name, t in got.items():
        T.check(t if name in ("last", "dstate") else turn(t), want[name], size[name], p["dtype"], name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [1, 2, 16, 33, 64, 65, 200, 515, 2000])
def test_lengths(L, dtype):
    _run(U.problem(L, 2, 2, L, 64, 64, dtype, state=True, dstate=True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("widths", [(1, 1), (64, 128), (128, 64), (128, 128), (96, 80), (33, 65), (7, 200), (256, 64), (64, 256), (250, 131)])
def test_widths(widths, dtype):
    _run(U.problem(3, 1, 2, 150, *widths, dtype, state=True, dstate=True))


@pytest.mark.parametrize("dtype,widths,heads", [("f32", (64, 64), 40), ("f32", (128, 48), 48), ("bf16", (96, 80), 30), ("bf16", (64, 64), 40), ("bf16", (33, 65), 30)])
def test_more_teams_than_compute_units(dtype, widths, heads):
    _run(U.problem(6, 2, heads, 130, *widths, dtype, lengths=[130, 97], state=True, dstate=True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layouts_and_lengths(dtype):
    _run(U.problem(4, 3, 3, 333, 64, 64, dtype, lengths=[333, 191, 0], state=True, dstate=True), layout="blhd")
    _run(U.problem(5, 2, 3, 140, 33, 65, dtype, lengths=[77, 140]), layout="blhd")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [0.02, 0.0, -1e-4, -1.0, -30.0])
def test_gates(gate, dtype):
    _run(U.problem(6, 1, 2, 170, 64, 64, dtype, gate=gate, state=True, dstate=True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gates_that_reset_now_and_then(dtype):
    p = U.problem(7, 2, 2, 200, 64, 64, dtype, state=True, dstate=True)
    p["a"][:, :, ::7] = float("-inf")
    p["a"][:, :, 3::11] = -3000.0
    _run(p)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("beta", [1.0, 2.0])
@pytest.mark.parametrize("same_key", [False, True])
def test_betas_and_keys_that_repeat(same_key, beta, dtype):
    _run(U.problem(8, 1, 2, 170, 64, 64, dtype, beta=beta, same_key=same_key, state=True, dstate=True, keys=1.0 if beta < 2 else 0.99), aligned=same_key)
