"""Inputs, oracle runs and tolerances of the tests of decayed linear attention."""
import numpy as np
import torch

from oracle import decay_oracle as D

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}

# Relative L2 error of a tensor.  A rounding to bf16 is off by at most u = 2^-8 of the value, by u / sqrt(3) in the root mean square.
# An output is a sum of terms of either sign; each term passes one rounding on its way (its weight inside a chunk, or the state that
# holds it), and the output one more: sqrt(2 / 3) u together, below u.  In fp32 (results of 32 bits: everything on fp32 inputs, the states
# on either) the chains of additions are at most 256 + 64 + the chunks' long: sqrt(512) 2^-24 / sqrt(3) < 2^-20, and the powers of g
# (exponent product and exponential) add 2^-22: below 2^-19.
L2 = {"f32": 2.0 ** -19, "bf16": 2.0 ** -8}
# Any element, against the same sum over absolute values: two roundings of 2^-8 for bf16; 1024 additions of 2^-24 for fp32.
ABS = {"f32": 2.0 ** -14, "bf16": 2.0 ** -7 * 1.01}


def problem(seed, B, H, L, dk, dv, dtype, *, decay=None, lengths=None, state=False, dstate=False):
    rng = np.random.default_rng(seed)

    def rows(d):
        x = torch.from_numpy(rng.standard_normal((B, H, L, d)).astype(np.float32)).to(TORCH[dtype])
        return x

    p = {"dtype": dtype, "Q": rows(dk), "K": rows(dk), "V": rows(dv), "dOut": rows(dv)}
    if decay is None:
        decay = np.log1p(-2.0 ** -np.linspace(2.0, 9.0, H)) if H > 1 else [-0.05]
    p["a"] = torch.tensor(np.resize(np.asarray(decay, dtype=np.float64), H), dtype=torch.float32)
    p["lengths"] = None if lengths is None else torch.tensor(np.resize(lengths, B), dtype=torch.int32)
    p["state"] = torch.from_numpy(rng.standard_normal((B, H, dk, dv)).astype(np.float32)) if state else None
    p["dstate"] = torch.from_numpy(rng.standard_normal((B, H, dk, dv)).astype(np.float32)) if dstate else None
    return p


def f64(t):
    return t.detach().double().cpu().numpy()


def oracle(p, scale=0.0, magnitude=False):
    """out, last, dQ, dK, dV, dstate in fp64; `magnitude`: of the absolute values of everything."""
    val = (lambda t: np.abs(f64(t))) if magnitude else f64
    Q, K, V, dO = (val(p[k]) for k in ("Q", "K", "V", "dOut"))
    B, H, L, dk = Q.shape
    dv = V.shape[3]
    scale = scale or dk ** -0.5
    zero = np.zeros((B, H, dk, dv))
    S, dS = (zero if p[k] is None else val(p[k]) for k in ("state", "dstate"))
    r = {k: np.zeros_like(x) for k, x in (("out", V), ("last", S), ("dQ", Q), ("dK", K), ("dV", V), ("dstate", S))}
    for b in range(B):
        n = L if p["lengths"] is None else min(max(int(p["lengths"][b]), 0), L)
        for h in range(H):
            a = float(p["a"][h])
            x = [t[b, h, :n] for t in (Q, K, V)]
            r["out"][b, h, :n], r["last"][b, h] = D.forward(*x, a, S[b, h], scale)
            r["dQ"][b, h, :n], r["dK"][b, h, :n], r["dV"][b, h, :n], r["dstate"][b, h] = D.backward(*x, a, S[b, h], scale, dO[b, h, :n], dS[b, h])
    return r


def check(got, want, size, dtype, what):
    """`got` against the oracle's `want`; `size`: the oracle's of absolute values."""
    g = f64(got)
    assert g.shape == want.shape, what
    assert np.isfinite(g).all(), what
    err = np.abs(g - want)
    norm = np.sqrt((want ** 2).sum())
    l2 = np.sqrt((err ** 2).sum()) / norm if norm > 0 else err.max(initial=0.0)
    worst = (err / np.maximum(size, 1e-300)).max(initial=0.0) if size.max(initial=0.0) > 0 else err.max(initial=0.0)
    print(f"{what}: L2 {l2:.2e} of {L2[dtype]:.2e}, element {worst:.2e} of {ABS[dtype]:.2e}")
    assert l2 <= L2[dtype], (what, l2)
    assert worst <= ABS[dtype], (what, worst)
