"""Inputs, oracle runs and tolerances of the tests of the gated delta rule."""
import numpy as np
import torch

from oracle import delta_oracle as D

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
ROWS = ("out", "dQ", "dK", "dV", "dlog_gate", "dbeta")

# Relative L2 error of a tensor.  A rounding to bf16 is off by at most u = 2^-8 of the value, by u / sqrt(3) in the root mean square.  An
# output is a sum of terms of either sign; each passes one rounding on its way (its weight inside a chunk), and the output one more:
# sqrt(2 / 3) u together, below u; gradients keep 16 bits on their way and are rounded once.  Results of 32 bits pass four products one after the
# other (K S, T R, K^T U and the inverse T), sums of at most 256 + 64 terms each: sqrt(320) 2^-24 / sqrt(3) < 2^-20.6 a product, 2^-19.6
# for four; truncated planes add 2^-23 a product, exponentials of sums of gates 2^-22; the correction of the state by later tokens
# shortens an error and never lengthens it (beta |k|^2 <= 2), so that a state has those of the chunks it remembers: below 2^-18 for ten of them.
L2 = {"f32": 2.0 ** -18, "bf16": 2.0 ** -8}
# A row's error, against the product of norms that bounds the terms of the row's sum (delta_oracle.py): the roundings of its operands are of that size.  Two roundings of
# 2^-8 for bf16; for 32 bits four products of 320 additions of 2^-24 in the worst order: 1280 2^-24 < 2^-13.
ROW = {"f32": 2.0 ** -13, "bf16": 2.0 ** -7 * 1.01}


def problem(seed, B, H, L, dk, dv, dtype, *, gate=None, beta=None, lengths=None, state=False, dstate=False, keys=1.0, same_key=False):
    rng = np.random.default_rng(seed)

    def rows(*shape):
        return torch.from_numpy(rng.standard_normal(shape).astype(np.float32))

    def unit(x):
        return x / x.norm(dim=-1, keepdim=True)

    p = {"dtype": dtype, "Q": unit(rows(B, H, L, dk)) if L else rows(B, H, L, dk), "K": rows(B, H, L, dk), "V": rows(B, H, L, dv), "dOut": rows(B, H, L, dv)}
    if L:
        p["K"] = keys * unit(p["K"][:, :, :1].expand(B, H, L, dk) if same_key else p["K"])
    for k in ("Q", "K", "V", "dOut"):
        p[k] = p[k].to(TORCH[dtype]).contiguous()
    e = torch.linspace(1.0, 9.0, H)[None, :, None] if H > 1 else torch.tensor(4.0)
    p["a"] = -torch.exp2(-e) * torch.exp(0.5 * rows(B, H, L)) if gate is None else torch.full((B, H, L), float(gate))
    p["beta"] = torch.sigmoid(1.5 * rows(B, H, L)) if beta is None else torch.full((B, H, L), float(beta))
    p["lengths"] = None if lengths is None else torch.tensor(np.resize(lengths, B), dtype=torch.int32)
    p["state"] = rows(B, H, dk, dv) if state else None
    p["dstate"] = rows(B, H, dk, dv) if dstate else None
    return p


def f64(t):
    return t.detach().double().cpu().numpy()


def oracle(p, scale=0.0):
    """(Results by name in fp64, the sizes of their rows)."""
    Q, K, V, dO, a, beta = (f64(p[k]) for k in ("Q", "K", "V", "dOut", "a", "beta"))
    B, H, L, dk = Q.shape
    dv = V.shape[3]
    scale = scale or dk ** -0.5
    zero = np.zeros((B, H, dk, dv))
    S, dS = (zero if p[k] is None else f64(p[k]) for k in ("state", "dstate"))
    r = {k: np.zeros_like(x) for k, x in (("out", V), ("last", S), ("dQ", Q), ("dK", K), ("dV", V), ("dlog_gate", a), ("dbeta", a), ("dstate", S))}
    size = {k: np.zeros((B, H, L)) for k in ROWS}
    size["last"], size["dstate"] = np.zeros((B, H)), np.zeros((B, H))
    for b in range(B):
        n = L if p["lengths"] is None else min(max(int(p["lengths"][b]), 0), L)
        for h in range(H):
            x = [t[b, h, :n] for t in (Q, K, V, a, beta)]
            r["out"][b, h, :n], r["last"][b, h], size["out"][b, h, :n], size["last"][b, h] = D.forward(*x, S[b, h], scale)
            g, s = D.backward(*x, S[b, h], scale, dO[b, h, :n], dS[b, h])
            for k, t in g.items():
                if k == "dstate":
                    r[k][b, h], size[k][b, h] = t, s[k]
                else:
                    r[k][b, h, :n], size[k][b, h, :n] = t, s[k]
    return r, size


def check(got, want, size, dtype, what, cancel=False):
    """`got` against the oracle's `want`; `size`: the sizes of its rows, or of its states.  `cancel`: keys so alike that
    the corrections of a chunk cancel one another (with one key and beta 1 a state is the last value, whatever the corrections before it): the
    error of such a sum is a share of its terms, whose norms `size` adds up, and not of what they leave."""
    g = f64(got)
    assert g.shape == want.shape, (what, g.shape, want.shape)
    assert np.isfinite(g).all(), what
    err = g - want
    total = np.sqrt((want ** 2).sum())
    if cancel or what in ("dlog_gate", "dbeta"):   # sums whose terms cancel
        total = np.sqrt((size ** 2).sum())
    if what in ("dlog_gate", "dbeta"):
        rows = np.abs(err)
    elif what in ("last", "dstate"):
        rows = np.sqrt((err ** 2).sum((-1, -2)))
    else:
        rows = np.sqrt((err ** 2).sum(-1))
    l2 = np.sqrt((err ** 2).sum()) / total if total > 0 else np.abs(err).max(initial=0.0)
    worst = (rows / np.maximum(size, 1e-30)).max(initial=0.0)
    print(f"{what}: L2 {l2:.2e} of {L2[dtype]:.2e}, row {worst:.2e} of {ROW[dtype]:.2e}")
    assert l2 <= L2[dtype], (what, l2)
    assert worst <= ROW[dtype], (what, worst)
