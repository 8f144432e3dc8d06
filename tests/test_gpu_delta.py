"""The gated delta rule: chunked forward, backward and single tokens against the fp64 oracle."""
import numpy as np
import pytest
import torch

import paper_2603_04127_amd as dk
from tests import delta_util as U

pytestmark = pytest.mark.gpu
NAMES = ("Q", "K", "V", "dOut", "a", "beta")
GRADS = {"dQ": "Q", "dK": "K", "dV": "V", "dlog_gate": "a", "dbeta": "beta", "dstate": "state"}


def _turn(t, layout):
    return t if layout == "bhld" or t is None else t.transpose(1, 2)


def _device(p, layout="bhld"):
    d = {k: _turn(p[k], layout).contiguous().cuda() for k in NAMES}
    d.update({k: None if p[k] is None else p[k].cuda() for k in ("lengths", "state", "dstate")})
    return d


def _forward(d, **kw):
    return dk.dark_delta_fwd(*(d[k] for k in ("Q", "K", "V", "a", "beta")), lengths=d["lengths"], state=d["state"], want_state=True, **kw)


def _backward(d, **kw):
    return dk.dark_delta_bwd(*(d[k] for k in ("Q", "K", "V", "a", "beta", "dOut")), lengths=d["lengths"], state=d["state"], dstate=d["dstate"], **kw)


def _check(p, got, layout="bhld", scale=0.0, ref=None, cancel=False):
    want, size = ref or U.oracle(p, scale)
    for k, t in got.items():
        state = k in ("last", "dstate")
        U.check(t if state else _turn(t, layout), want[k], size[k], "f32" if state or k in ("dlog_gate", "dbeta") else p["dtype"], k, cancel or p["Q"].shape[3] == 1)


def _run(p, layout="bhld", scale=0.0, cancel=False):
    d = _device(p, layout)
    out, last = _forward(d, layout=layout, scale=scale)
    g = _backward(d, layout=layout, scale=scale)
    torch.cuda.synchronize()
    _check(p, {"out": out, "last": last, **g}, layout, scale, cancel=cancel)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [1, 2, 15, 16, 17, 31, 33, 64, 65, 200, 515])
def test_lengths(L, dtype):
    _run(U.problem(L, 2, 3, L, 64, 64, dtype, state=True, dstate=True))
    _run(U.problem(L + 1, 1, 2, L, 64, 64, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("widths", [(1, 1), (64, 128), (128, 64), (128, 128), (96, 80), (33, 65), (7, 200), (256, 64), (64, 256), (256, 256), (250, 131)])
def test_widths(widths, dtype):
    _run(U.problem(3, 1, 2, 150, *widths, dtype, state=True, dstate=True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["bhld", "blhd"])
def test_layouts_and_ragged_batches(layout, dtype):
    _run(U.problem(4, 2, 3, 333, 64, 64, dtype, lengths=[333, 191], state=True, dstate=True), layout)
    _run(U.problem(5, 1, 2, 260, 40, 72, dtype), layout)
    _run(U.problem(5, 2, 3, 140, 33, 65, dtype, lengths=[77, 140], state=True), layout)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [0.02, 0.0, -1e-4, -1.0, -30.0, -1e5, -np.inf])
def test_gates(gate, dtype):
    _run(U.problem(6, 1, 2, 170, 64, 64, dtype, gate=gate, state=True, dstate=True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gates_that_reset_now_and_then(dtype):
    # what is remembered behind a reset is as exact as before it: sums of gates keep 48 bits
    p = U.problem(7, 2, 2, 200, 64, 64, dtype, state=True, dstate=True)
    p["a"][:, :, ::7] = float("-inf")
    p["a"][:, :, 3::11] = -3000.0
    p["a"][:, :, 5::13] = -90.0
    _run(p)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("beta", [0.0, 1.0, 2.0])
@pytest.mark.parametrize("same_key", [False, True])
def test_betas_and_keys_that_repeat(same_key, beta, dtype):
    # one key throughout couples all of a chunk's tokens: the triangle's inverse is as far from the identity as it gets
    _run(U.problem(8, 1, 2, 170, 64, 64, dtype, beta=beta, same_key=same_key, state=True, dstate=True, keys=1.0 if beta < 2 else 0.99), cancel=same_key)


@pytest.mark.parametrize("keys", [2.0 ** -40, 2.0 ** -10])
def test_small_keys(keys):
    for dtype in ("f32", "bf16"):
        _run(U.problem(9, 1, 2, 100, 64, 64, dtype, keys=keys, state=True, dstate=True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths", [[0, 1, 64, 140], [140, 65, 0, 63], [-3, 1000, 128, 127]])
def test_ragged_batches_read_nothing_behind_a_sequence(lengths, dtype):
    p = U.problem(10, 4, 2, 140, 64, 64, dtype, lengths=lengths, state=True, dstate=True)
    for b in range(4):
        for k in NAMES:
            p[k][b, :, min(max(lengths[b], 0), 140):] = 0.0
    ref = U.oracle(p)
    d = _device(p)
    for b in range(4):
        for k, bad in zip(NAMES, (float("nan"), float("inf"), float("-inf"), float("nan"), float("inf"), float("nan"))):
            d[k][b, :, min(max(lengths[b], 0), 140):] = bad
    out, last = _forward(d)
    g = _backward(d)
    torch.cuda.synchronize()
    _check(p, {"out": out, "last": last, **g}, ref=ref)
    for b in range(4):
        for t in (out, *(t for k, t in g.items() if k != "dstate")):
            assert (t[b, :, min(max(lengths[b], 0), 140):] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["bhld", "blhd"])
@pytest.mark.parametrize("widths", [(33, 65), (1, 3), (66, 31), (150, 7)])
def test_odd_widths_touch_nothing_beside_them(widths, layout, dtype):
    lengths = [130, 67, 0, 129]
    p = U.problem(14, 4, 3, 130, *widths, dtype, lengths=lengths, state=True, dstate=True)
    for k in NAMES:
        for b in range(4):
            p[k][b, :, lengths[b]:] = 0.0
    ref = U.oracle(p)
    d = _device(p, layout)
    for k in NAMES:
        for b in range(4):
            _turn(d[k], layout)[b, :, lengths[b]:] = float("nan")
    room = []

    def inside(t):   # a tensor of t's kind, 256 elements into a larger one
        room.append(torch.full((t.numel() + 512,), 7.0, dtype=t.dtype, device="cuda"))
        return room[-1][256:256 + t.numel()].view(t.shape)

    out, last = inside(d["V"]), inside(d["state"])
    grads = {k: inside(d[x]) for k, x in GRADS.items()}
    _forward(d, layout=layout, out=out, state_out=last)
    _backward(d, layout=layout, grads=grads)
    torch.cuda.synchronize()
    _check(p, {"out": out, "last": last, **grads}, layout, ref=ref)
    assert all((r[:256] == 7).all() and (r[-256:] == 7).all() for r in room)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows_pass_the_state_on(dtype):
    d = _device(U.problem(11, 2, 2, 0, 64, 48, dtype, state=True, dstate=True))
    out, last = _forward(d)
    g = _backward(d)
    assert out.shape == (2, 2, 0, 48) and torch.equal(last, d["state"]) and torch.equal(g["dstate"], d["dstate"])
    d["state"] = None
    assert (_forward(d)[1] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_gate_is_a_gate_of_zero(dtype):
    p = U.problem(12, 2, 2, 150, 64, 32, dtype, gate=0.0, state=True, dstate=True)
    d = _device(p)
    want = (*_forward(d), *_backward(d).values())
    d["a"] = None
    g = _backward(d)
    assert "dlog_gate" not in g
    assert all(torch.equal(x, y) for x, y in zip((*_forward(d), *g.values()), want[:6] + want[7:]))


@pytest.mark.parametrize("dtype,widths,B", [("bf16", (64, 64), 1), ("bf16", (128, 128), 7), ("bf16", (33, 65), 1), ("f32", (64, 64), 1), ("f32", (31, 33), 1)])
def test_gradients_one_by_one(dtype, widths, B):
    d = _device(U.problem(21, B, 3, 200, *widths, dtype, state=True, dstate=True))
    want = _backward(d)
    for name, t in want.items():
        alone = _backward(d, need=(name,))
        assert list(alone) == [name] and torch.equal(alone[name], t), name


def test_state_in_place_and_continued_prompts():
    p = U.problem(13, 2, 2, 300, 64, 64, "bf16", state=True)
    d = _device(p)
    ref = U.oracle(p)
    S = d["state"].clone()
    got, same = dk.dark_delta_fwd(*(d[k] for k in ("Q", "K", "V", "a", "beta")), state=S, state_out=S)
    assert same is S
    _check(p, {"out": got, "last": S}, ref=ref)
    part = lambda a, b: [d[k][:, :, a:b].contiguous() for k in ("Q", "K", "V", "a", "beta")]
    first, S = dk.dark_delta_fwd(*part(0, 111), state=d["state"], want_state=True)   # the same prompt in two calls
    second, S = dk.dark_delta_fwd(*part(111, 300), state=S, want_state=True)
    _check(p, {"out": torch.cat([first, second], 2), "last": S}, ref=ref)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("widths", [(64, 64), (128, 64), (33, 65)])
def test_the_same_bits_whatever_is_handed_out(widths, dtype):
    d = _device(U.problem(15, 2, 3, 333, *widths, dtype, lengths=[333, 191]))
    out, grads = _forward(d)[0], _backward(d)
    assert torch.equal(dk.dark_delta_fwd(*(d[k] for k in ("Q", "K", "V", "a", "beta")), lengths=d["lengths"]), out)
    for need in (("dQ",), ("dK",), ("dV",), ("dlog_gate",), ("dbeta",), ("dK", "dbeta")):
        got = _backward(d, need=need)
        assert set(got) == set(need) and all(torch.equal(got[k], grads[k]) for k in need)
    d["state"] = d["dstate"] = torch.zeros(2, 3, *widths, device="cuda")   # an empty state is none
    assert torch.equal(_forward(d)[0], out)
    same = _backward(d)
    assert "dstate" in same and all(torch.equal(same[k], t) for k, t in grads.items())
    assert torch.equal(_backward(d, need=("dstate",))["dstate"], same["dstate"])


def test_scale_and_repeatability():
    p = U.problem(16, 2, 4, 500, 64, 64, "bf16", state=True, dstate=True)
    _run(p, scale=0.75)
    d = _device(p)
    a, b = (_forward(d) + tuple(_backward(d).values()) for _ in range(2))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_are_the_differences_of_the_forward(dtype):
    # the kernels' own forward, on either side of a step along a direction; the loss in 64 bits.  A difference quotient of step e is off
    # by the forward's error over e and by e^2 of the third derivative: 2^-18 of the loss's terms over 2^-5, and 2^-10.
    p = U.problem(17, 1, 2, 150, 32, 32, "f32", state=True, dstate=True)
    d = _device(p)
    g = _backward({**d, **{k: d[k].to(U.TORCH[dtype]) for k in ("Q", "K", "V", "dOut")}})

    def loss(x):
        out, last = _forward(x)
        return float((out.double() * d["dOut"].double()).sum() + (last.double() * d["dstate"].double()).sum())

    gen = torch.Generator(device="cuda").manual_seed(1)
    for name, key in GRADS.items():
        step = torch.randn(d[key].shape, generator=gen, device="cuda")
        step *= 2.0 ** -5 * d[key].norm() / step.norm()
        num = loss({**d, key: d[key] + step}) - loss({**d, key: d[key] - step})
        ana = float((2 * step.double() * g[name].double()).sum())
        bound = float(2 * step.double().norm() * g[name].double().norm())
        assert abs(num - ana) <= (2.0 ** -7 if dtype == "f32" else 2.0 ** -6) * bound, (name, num, ana, bound)


def test_infinity_and_nan_stay_behind_their_chunk():
    for dtype, C in (("f32", 32), ("bf16", 64)):
        d = _device(U.problem(18, 1, 1, 300, 64, 64, dtype))
        clean = _forward(d)[0]
        for name, bad in (("K", float("nan")), ("K", float("inf")), ("V", float("inf")), ("a", float("nan")), ("beta", float("nan"))):
            e = {**d, name: d[name].clone()}
            e[name][(0, 0, 200, 3) if name in "KV" else (0, 0, 200)] = bad
            out = _forward(e)[0]
            assert torch.equal(out[:, :, :200 // C * C], clean[:, :, :200 // C * C])
            assert not torch.isfinite(out[0, 0, 200:, 3]).any(), (dtype, name)
        e = {**d, "Q": d["Q"].clone()}
        e["Q"][0, 0, 200, 3] = float("nan")
        out = _forward(e)[0]
        out[0, 0, 200] = clean[0, 0, 200]
        assert torch.equal(out, clean)


# ---------------------------------------------------------------------------
# single tokens
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 3, 64, 64), (1, 1, 1, 1), (3, 2, 33, 65), (1, 2, 256, 256), (2, 2, 128, 20), (70, 16, 128, 128), (1, 5, 100, 200), (2, 1, 200, 7)])
def test_steps_are_the_forward(shape, dtype):
    B, H, dkey, dval = shape
    p = U.problem(20, B, H, 3 if B * H > 100 else 20, dkey, dval, dtype, state=True)
    d = _device(p)
    S = d["state"].clone()
    out = torch.stack([dk.dark_delta_step(*(d[k][:, :, t].contiguous() for k in ("Q", "K", "V", "a", "beta")), S) for t in range(p["Q"].shape[2])], 2)
    _check(p, {"out": out, "last": S})


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_steps_from_parents(dtype):
    p = U.problem(21, 6, 2, 1, 48, 72, dtype)
    d = _device(p)
    past = torch.randn(4, 2, 48, 72, device="cuda")
    parent = torch.tensor([3, 0, 0, -1, 4, 2], dtype=torch.int32, device="cuda")   # -1 and 4 are no rows: empty states
    S = torch.full((6, 2, 48, 72), float("nan"), device="cuda")
    before = past.clone()
    one = [d[k][:, :, 0].contiguous() for k in ("Q", "K", "V", "a", "beta")]
    out = dk.dark_delta_step(*one, past, parent=parent, state_out=S)
    p["state"] = torch.stack([past[r].cpu() if 0 <= r < 4 else torch.zeros(2, 48, 72) for r in parent.tolist()])
    _check(p, {"out": out[:, :, None], "last": S})
    assert torch.equal(past, before)
    T = torch.empty_like(S)
    same = dk.dark_delta_step(*one[:3], None, one[4], past, parent=parent, state_out=T)
    assert torch.equal(same, dk.dark_delta_step(*one[:3], torch.zeros_like(one[3]), one[4], past, parent=parent, state_out=S)) and torch.equal(S, T)


# ---------------------------------------------------------------------------
# streams and graphs
# ---------------------------------------------------------------------------
def _all(d):
    return (*_forward(d), *_backward(d).values())


def test_two_streams_at_once():
    ds = [_device(U.problem(30 + i, 1, 4, 1000, 64, 64, "bf16", state=True, dstate=True)) for i in range(2)]
    want = [_all(d) for d in ds]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ds]
    for _ in range(3):
        got = []
        for d, s in zip(ds, streams):
            with torch.cuda.stream(s):
                got.append(_all(d))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for g, w in zip(got, want) for x, y in zip(g, w))


def test_two_threads_at_once():
    import threading

    ds = [_device(U.problem(32 + i, 1, 4, 700, 64, 64, "bf16", state=True, dstate=True)) for i in range(2)]
    want = [_all(d) for d in ds]
    torch.cuda.synchronize()
    got = [None, None]

    def run(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                got[i] = _all(ds[i])
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert all(torch.equal(x, y) for g, w in zip(got, want) for x, y in zip(g, w))


def test_two_graphs_replay_in_turn():
    ds = [_device(U.problem(40 + i, 1, 4, L, 64, 64, "bf16", state=True, dstate=True)) for i, L in enumerate((60, 900))]

    def work(d):   # the state is updated in place from a copy, so that a replay starts from the same one
        S = d["state"].clone()
        one = [d[k][:, :, 0].contiguous() for k in ("Q", "K", "V", "a", "beta")]
        out, _ = dk.dark_delta_fwd(*(d[k] for k in ("Q", "K", "V", "a", "beta")), state=S, state_out=S)
        T = S.clone()
        return (out, S, *_backward(d).values(), dk.dark_delta_step(*one, T), T)

    for d in ds:
        work(d)
    torch.cuda.synchronize()
    graphs, held = [], []
    for d in ds:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            held.append(work(d))
    for i in range(4):
        for d in ds:
            for k in ("Q", "V", "state", "dstate", "dOut"):
                d[k].copy_(torch.randn_like(d[k]))
        for j in ((0, 1), (1, 0))[i % 2]:
            graphs[j].replay()
        torch.cuda.synchronize()
        got = [[t.clone() for t in h] for h in held]
        assert all(torch.equal(x, y) for g, d in zip(got, ds) for x, y in zip(g, work(d)))


# ---------------------------------------------------------------------------
# a sequence's results, bit by bit, beside few others and beside more than there are compute units
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,dk_,dv", [("f32", 64, 64), ("f32", 128, 128), ("f32", 48, 56), ("f32", 31, 33), ("bf16", 64, 64), ("bf16", 128, 128), ("bf16", 96, 80),
                                          ("bf16", 33, 65), ("bf16", 64, 72), ("bf16", 256, 64)])
def test_results_do_not_depend_on_the_batch(dtype, dk_, dv):
    B, H, L = 24, 4, 150
    g = torch.Generator(device="cuda").manual_seed(8)
    q, k, v, o = (torch.randn(B, H, L, d, generator=g, device="cuda") for d in (dk_, dk_, dv, dv))
    q, k, v, o = (x.to(U.TORCH[dtype]) for x in (q / 8, k / k.norm(dim=-1, keepdim=True), v, o))
    a, beta = -0.1 * torch.rand(B, H, L, generator=g, device="cuda"), torch.rand(B, H, L, generator=g, device="cuda")
    lengths = torch.randint(0, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    state, dstate = (torch.randn(B, H, dk_, dv, generator=g, device="cuda") for _ in range(2))
    out, last = dk.dark_delta_fwd(q, k, v, a, beta, lengths=lengths, state=state, want_state=True)
    grads = dk.dark_delta_bwd(q, k, v, a, beta, o, lengths=lengths, state=state, dstate=dstate)
    for b in (0, B - 1):
        q1, k1, v1, a1, b1, o1, n1, s1, d1 = (x[b:b + 1].clone() for x in (q, k, v, a, beta, o, lengths, state, dstate))
        out1, last1 = dk.dark_delta_fwd(q1, k1, v1, a1, b1, lengths=n1, state=s1, want_state=True)
        assert torch.equal(out[b:b + 1], out1) and torch.equal(last[b:b + 1], last1)
        for name, x in dk.dark_delta_bwd(q1, k1, v1, a1, b1, o1, lengths=n1, state=s1, dstate=d1).items():
            assert torch.equal(grads[name][b:b + 1], x), name


# ---------------------------------------------------------------------------
# tensors of more than 2^32 bytes: the last sequence against a call of its own
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("layout", ["bhld", "blhd"])
@pytest.mark.parametrize("dtype,L", [("bf16", 8000), ("f32", 2000)])
def test_offsets_beyond_32_bits(dtype, L, layout):
    H, d = 16, 128
    B = (1 << 32) // (H * L * d * (2 if dtype == "bf16" else 4)) + 2
    shape = (B, H, L, d) if layout == "bhld" else (B, L, H, d)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = [torch.zeros(shape, dtype=U.TORCH[dtype], device="cuda") for _ in range(4)]
    for t in x:
        t[-1] = torch.randn(shape[1:], generator=g, device="cuda") / (8.0 if t is x[1] else 1.0)
    a = -0.1 * torch.rand(shape[:3], generator=g, device="cuda")
    beta = torch.rand(shape[:3], generator=g, device="cuda")
    out, state = dk.dark_delta_fwd(*x[:3], a, beta, want_state=True, layout=layout)
    grads = dk.dark_delta_bwd(*x[:3], a, beta, x[3], state=state, layout=layout)
    alone = [t[-1:].clone() for t in (*x, a, beta)]
    want, last = dk.dark_delta_fwd(*alone[:3], *alone[4:], want_state=True, layout=layout)
    assert torch.equal(out[-1:], want) and torch.equal(state[-1:], last) and not out[0].any()
    for name, t in dk.dark_delta_bwd(*alone[:3], *alone[4:], alone[3], state=last, layout=layout).items():
        assert torch.equal(grads[name][-1:], t), name


def test_step_offsets_beyond_32_bits():
    B, H, d = 1026, 16, 256
    g = torch.Generator(device="cuda").manual_seed(6)
    past, S = (torch.zeros(B, H, d, d, device="cuda") for _ in range(2))
    past[-1] = torch.randn(H, d, d, generator=g, device="cuda")
    q, k, v = (torch.randn(B, H, d, generator=g, device="cuda") / 16 for _ in range(3))
    a, beta = -torch.rand(B, H, generator=g, device="cuda"), torch.rand(B, H, generator=g, device="cuda")
    parent = torch.zeros(B, dtype=torch.int32, device="cuda")
    parent[-1] = B - 1
    out = dk.dark_delta_step(q, k, v, a, beta, past, parent=parent, state_out=S)
    D = torch.exp(a[-1].double())[:, None, None] * past[-1].double()
    u = beta[-1].double()[:, None] * (v[-1].double() - (D * k[-1].double()[:, :, None]).sum(1))
    want = D + k[-1].double()[:, :, None] * u[:, None]
    assert torch.allclose(S[-1].double(), want, rtol=1e-6, atol=1e-6)
    assert torch.allclose(out[-1].double(), (want * q[-1].double()[:, :, None]).sum(1) / 16, rtol=1e-5, atol=1e-5)
