"""Tokens drawn from logits against the fp64 oracle, and a decoding loop over states of the gated delta rule."""
import numpy as np
import pytest
import torch

import paper_2603_04127_amd as dk
from oracle import delta_oracle, sample_oracle as S

pytestmark = pytest.mark.gpu
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}

# A weight is off by a few units of the last place (a unit of 2^-23 of the exponential, one of the product), sums are in 64 bits: shares of a
# row are off by less than 2^-20, and so is the logarithm of one beside its own rounding of 2^-24 of its value.  A random number closer
# than 2^-20 to a border between two tokens may draw either, and so may one where the border of top_p lies that close to a token's: such
# rows are not drawn here (about one of 2^20 times the number of kept tokens).
NEAR = 2.0 ** -20


def _logits(rng, B, V, dtype, spread=2.5):
    return torch.from_numpy((spread * rng.standard_normal((B, V))).astype(np.float32)).to(TORCH[dtype])


def _run(x, u, **kw):
    B = x.shape[0]
    per_row = {k: np.broadcast_to(np.asarray(v), (B,)) for k, v in kw.items()}
    tensors = {k: torch.tensor(v.copy(), dtype=torch.int32 if k == "top_k" else torch.float32).cuda() if np.ndim(kw[k]) else kw[k] for k, v in per_row.items()}
    token, log = dk.dark_sample(x.cuda(), None if u is None else torch.from_numpy(u).cuda(), want_logprob=True, **tensors)
    token, log = token.cpu().numpy(), log.double().cpu().numpy()
    rows = x.double().numpy()
    for b in range(B):
        args = {k: float(np.float32(v[b])) if k != "top_k" else int(v[b]) for k, v in per_row.items()}
        t, l, near = S.draw(rows[b], 0.0 if u is None else float(u[b]), **args)
        w = S.kept(rows[b], **{**dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **args})
        if token[b] != t:
            # only where u is on a border: the token drawn is the neighbour behind or before it among those that are kept
            assert near <= NEAR, (b, token[b], t, near, args)
            continue
        assert l == -np.inf and log[b] == l or abs(log[b] - l) <= NEAR + 2.0 ** -23 * abs(l), (b, log[b], l)
        assert t < 0 or w[t] > 0
    return token


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 63, 64, 65, 1000, 4097, 32000, 65537])
def test_sizes(V, dtype):
    rng = np.random.default_rng(V)
    x, u = _logits(rng, 5, V, dtype), rng.random(5).astype(np.float32)
    for kw in (dict(), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=1), dict(temperature=0.0), dict(temperature=0.7, top_k=40, top_p=0.8, min_p=0.02),
               dict(top_k=600, top_p=0.95), dict(top_k=600), dict(top_p=0.999), dict(top_k=V), dict(top_k=V - 1, top_p=0.5)):
        _run(x, u, **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_rows_with_settings_of_their_own(dtype):
    rng = np.random.default_rng(1)
    B, V = 24, 131071 if dtype == "bf16" else 262147
    x, u = _logits(rng, B, V, dtype), rng.random(B).astype(np.float32)
    _run(x, u, temperature=np.where(rng.random(B) < 0.1, 0.0, 0.5 + rng.random(B)), top_k=np.where(rng.random(B) < 0.5, 0, rng.integers(1, 3000, B)),
         top_p=np.where(rng.random(B) < 0.3, 1.0, 0.5 + 0.5 * rng.random(B)), min_p=np.where(rng.random(B) < 0.5, 0.0, 0.1 * rng.random(B)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_token_in_its_turn(dtype):
    # random numbers in the middle of every kept token's share draw that token: nothing is skipped, at lanes', waves' and parts' ends alike
    rng = np.random.default_rng(2)
    x = _logits(rng, 1, 700, dtype, 0.5)
    w = S.kept(x.double().numpy()[0], 1.0, 0, 0.9, 0.0)
    at = np.nonzero(w)[0]
    sums = np.cumsum(w[at]) / w.sum()
    u = (sums - 0.5 * w[at] / w.sum()).astype(np.float32)
    token = _run(x.expand(at.size, -1).contiguous(), u, top_p=0.9)
    assert (token == at).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_logits(dtype):
    # ties by the token's number: all equal, two values, and rows of a few values whose bins hold more than is sorted at once
    rng = np.random.default_rng(3)
    u = rng.random(6).astype(np.float32)
    for V in (100, 5000, 50000):
        for x in (torch.zeros(6, V), torch.from_numpy((rng.integers(0, 2, (6, V))).astype(np.float32)), torch.from_numpy(rng.integers(0, 5, (6, V)).astype(np.float32) / 4)):
            x = x.to(TORCH[dtype])
            for kw in (dict(), dict(top_k=37), dict(top_k=3000), dict(top_p=0.37), dict(top_p=0.83, top_k=4000), dict(temperature=0.0), dict(top_k=1)):
                _run(x, u, **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_logits(dtype):
    rng = np.random.default_rng(4)
    V = 3000
    lowest = torch.finfo(TORCH[dtype]).min
    x = _logits(rng, 9, V, dtype)
    x[0] = float("-inf")
    x[1] = float("nan")
    x[2, 1:] = float("-inf")
    x[3, ::2] = float("nan")
    x[4, :] = lowest
    x[5, 5:] = lowest
    x[6, [7, 2900]] = float("inf")
    x[7, 17] = float("inf")
    x[7, 18] = float("nan")
    x[8, 100:] = float("-inf")
    if dtype == "bf16":
        x.view(torch.int16)[3, ::4] = 0x7f81   # a NaN that signals
    u = rng.random(9).astype(np.float32)
    for kw in (dict(), dict(top_k=20), dict(top_k=1000), dict(top_p=0.9), dict(min_p=0.1), dict(temperature=0.0), dict(top_k=1500, top_p=0.7), dict(top_k=150, top_p=0.7)):
        token = _run(x, u, **kw)
        assert token[0] == token[1] == -1 and token[2] == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_shares_of_very_long_rows(dtype):
    # Tokens of 1e-7 of the sum each: the share before and behind the drawn one says more than its number.  Where top_p is looked for a weight is off
    # by half a unit of 2^-36 of the largest at most, 2^25 of them by 2^-12; their sum is more than 100 times the largest: 2.4e-6 of it, twice that for
    # the whole and the part.
    V, tol = (1 << 25) + 1, 5e-6
    g = torch.Generator(device="cuda").manual_seed(15)
    x = (3.0 * torch.randn(1, V, generator=g, device="cuda")).to(TORCH[dtype])
    z, at = torch.sort(x[0].float(), descending=True, stable=True)
    e = torch.exp(z.double() - z[0].double())
    assert e.sum() > 100
    for u, p, q in ((0.3, 0.9, 0.0), (0.85, 0.9, 0.0), (0.5, 0.999, 0.0), (0.6, 0.9, 1e-5), (0.25, 1.0, 0.0)):
        t = int(dk.dark_sample(x, torch.full((1,), u, device="cuda"), top_p=p, min_p=q))
        n = V if p >= 1.0 else int((torch.cumsum(e, 0) - e < float(np.float32(p)) * e.sum()).sum())
        w = torch.zeros(V, dtype=torch.float64, device="cuda")
        w[at[:n]] = torch.where(e[:n] >= float(np.float32(q)), e[:n], 0.0)
        c = torch.cumsum(w, 0)
        share = c[t] / c[-1], (c[t] - w[t]) / c[-1]
        assert share[0] >= u - tol and share[1] <= u + tol, (u, p, q, float(share[0]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_without_filters_weighed_on_the_way(dtype):
    # a row's first logits say little about the others: masked, far below or far above them, all alike
    rng = np.random.default_rng(14)
    V = 70001
    x = _logits(rng, 9, V, dtype)
    x[0, :40000] = float("-inf")
    x[1, :60000] -= 5e3
    x[2, 5000:] -= 5e3
    x[3, 1:] = float("-inf")
    x[4, :-1] = float("-inf")
    x[5] = torch.linspace(-2e4, 2e4, V)
    x[6] = torch.linspace(2e4, -2e4, V)
    x[7, 30000] = float("inf")
    x[8] = 0.0
    u = np.array([0.3, 0.999, 0.5, 0.5, 0.5, 0.7, 0.1, 0.9, 0.4], dtype=np.float32)
    for kw in (dict(), dict(temperature=0.01), dict(temperature=30.0), dict(temperature=1e-6), dict(temperature=np.linspace(0.0, 2.0, 9))):
        _run(x, u, **kw)


def test_settings_at_their_ends():
    rng = np.random.default_rng(5)
    x = _logits(rng, 4, 2000, "f32")
    u = np.array([0.0, 0.25, 1.0 - 2.0 ** -24, 1.0], dtype=np.float32)
    for kw in (dict(top_p=0.0), dict(top_p=-1.0), dict(top_p=1e-30), dict(min_p=1.0), dict(min_p=5.0), dict(top_p=2.0), dict(min_p=-1.0), dict(top_k=-5),
               dict(temperature=1e-4), dict(temperature=1e-30), dict(temperature=1e4), dict(temperature=1e30), dict(top_p=1.0 - 2.0 ** -24), dict(temperature=1e-3, top_k=1000),
               dict(temperature=50.0, top_p=0.5)):
        _run(x, u, **kw)
    for bad in (np.array([-1.0, float("nan"), -0.0, 3.0], dtype=np.float32),):   # outside 0 ... 1: the nearer end
        token = dk.dark_sample(x.cuda(), torch.from_numpy(bad).cuda()).cpu().numpy()
        assert (token[:3] == 0).all() and token[3] == 1999
    nan = torch.full((4,), float("nan"), device="cuda")
    assert torch.equal(dk.dark_sample(x.cuda(), torch.from_numpy(u).cuda(), top_p=nan, min_p=nan), dk.dark_sample(x.cuda(), torch.from_numpy(u).cuda()))
    assert (dk.dark_sample(x.cuda(), torch.from_numpy(u).cuda(), temperature=nan).cpu() == x.argmax(1)).all()


def test_rows_beside_each_other_and_given_results():
    # odd rows begin anywhere; the results' neighbours stay as they are; the same bits in every call
    rng = np.random.default_rng(6)
    x, u = _logits(rng, 7, 1001, "bf16").cuda(), torch.from_numpy(rng.random(7).astype(np.float32)).cuda()
    room = torch.full((9,), -7, dtype=torch.int32, device="cuda")
    got = dk.dark_sample(x, u, top_p=0.9, out=room[1:8])
    assert got.data_ptr() == room[1:8].data_ptr() and room[0] == -7 and room[8] == -7
    for b in range(7):
        assert dk.dark_sample(x[b:b + 1].clone(), u[b:b + 1].clone(), top_p=0.9) == got[b]
    assert all(torch.equal(dk.dark_sample(x, u, top_p=0.9), got) for _ in range(5))
    assert dk.dark_sample(x[:0], u[:0]).shape == (0,)


def test_how_often_tokens_are_drawn():
    # 20,000 random numbers: shares within six standard deviations
    rng = np.random.default_rng(7)
    n = 20000
    x = _logits(rng, 1, 40, "f32", 1.0)
    w = S.kept(x.double().numpy()[0], 0.8, 20, 0.95, 0.0)
    p = w / w.sum()
    u = torch.from_numpy(rng.random(n).astype(np.float32)).cuda()
    token = dk.dark_sample(x.expand(n, -1).contiguous().cuda(), u, temperature=0.8, top_k=20, top_p=0.95).cpu().numpy()
    share = np.bincount(token, minlength=40) / n
    assert (np.abs(share - p) <= 6 * np.sqrt(p * (1 - p) / n) + 1e-6).all()


def test_streams_and_graphs():
    rng = np.random.default_rng(8)
    x = [_logits(rng, 8, 9000, "bf16").cuda() for _ in range(2)]
    u = [torch.from_numpy(rng.random(8).astype(np.float32)).cuda() for _ in range(2)]
    want = [dk.dark_sample(a, b, top_k=30, want_logprob=True) for a, b in zip(x, u)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in x]
    for _ in range(3):
        got = []
        for a, b, s in zip(x, u, streams):
            with torch.cuda.stream(s):
                got.append(dk.dark_sample(a, b, top_k=30, want_logprob=True))
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for g, w in zip(got, want) for p, q in zip(g, w))
    hx, hu = x[0].clone(), u[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = dk.dark_sample(hx, hu, top_k=30, want_logprob=True)
    for i in range(4):
        hx.copy_(x[i % 2])
        hu.copy_(u[i % 2])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held, want[i % 2]))
        dk.dark_sample(x[1], u[1], top_p=0.5)   # eager work between the replays


def test_offsets_beyond_32_bits():
    V = 131071
    B = (1 << 32) // (2 * V) + 3
    x = torch.zeros(B, V, dtype=torch.bfloat16, device="cuda")
    x[-1, 70001] = 30.0
    x[-2, V - 1] = 30.0
    u = torch.full((B,), 0.5, device="cuda")
    token = dk.dark_sample(x, u)
    assert token[-1] == 70001 and token[-2] == V - 1 and token[0] == V // 2


def test_a_prompt_and_a_decoding_loop():
    # as a program decodes: the prompt by the chunked form, then token by token, each drawn from logits of the layer's output; the states of
    # the sequences that are carried on are picked by their parents in the middle of it.  Against the same loop by the oracles.
    B, H, L, d, V, steps = 3, 2, 70, 32, 500, 12
    g = torch.Generator().manual_seed(9)
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)
    emb = {k: torch.randn(V, H, d, generator=g) for k in ("q", "k", "v")}
    emb["q"], emb["k"] = unit(emb["q"]), unit(emb["k"])
    gate, beta = -0.2 * torch.rand(V, H, generator=g), torch.sigmoid(torch.randn(V, H, generator=g))
    head = torch.randn(H * d, V, generator=g)
    prompt = torch.randint(0, V, (B, L), generator=g)
    uniform = torch.rand(steps, B, generator=g)
    setting = dict(temperature=0.9, top_k=40, top_p=0.9, min_p=0.01)
    parent = torch.tensor([2, 0, 0])
    dev = lambda t: t.cuda().contiguous()
    Q, K, Vv = (dev(emb[k][prompt].transpose(1, 2)) for k in ("q", "k", "v"))
    out, state = dk.dark_delta_fwd(Q, K, Vv, dev(gate[prompt].transpose(1, 2)), dev(beta[prompt].transpose(1, 2)), want_state=True)
    last = out[:, :, -1]
    f64 = lambda t: t.double().numpy()
    ref_state, ref_last = np.zeros((B, H, d, d)), np.zeros((B, H, d))
    for b in range(B):
        for h in range(H):
            x = [f64(emb[k][prompt[b], h]) for k in ("q", "k", "v")] + [f64(t[prompt[b], h]) for t in (gate, beta)]
            o, ref_state[b, h], _, _ = delta_oracle.forward(*x, np.zeros((d, d)), d ** -0.5)
            ref_last[b, h] = o[-1]
    seen = []
    for i in range(steps):
        logits = (last.reshape(B, H * d) @ dev(head)).contiguous()
        token = dk.dark_sample(logits, dev(uniform[i]), **setting)
        ref_logits = ref_last.reshape(B, H * d) @ f64(head)
        ref = [S.draw(ref_logits[b], float(uniform[i, b]), **{k: float(np.float32(v)) if k != "top_k" else v for k, v in setting.items()}) for b in range(B)]
        assert all(r[2] > 1e-4 for r in ref)   # no border near: the logits are fp32 sums
        assert token.cpu().tolist() == [r[0] for r in ref]
        seen.append(token.cpu().tolist())
        t = token.cpu().long()
        step = [dev(emb[k][t]) for k in ("q", "k", "v")] + [dev(gate[t]), dev(beta[t])]
        if i == steps // 2:
            old, state = state, torch.empty_like(state)
            last = dk.dark_delta_step(*step, old, parent=dev(parent.int()), state_out=state)
            ref_state = ref_state[parent.numpy()]
        else:
            last = dk.dark_delta_step(*step, state)
        for b in range(B):
            for h in range(H):
                x = [f64(emb[k][t[b], h])[None] for k in ("q", "k", "v")] + [f64(a[t[b], h])[None] for a in (gate, beta)]
                o, ref_state[b, h], _, _ = delta_oracle.forward(*x, ref_state[b, h], d ** -0.5)
                ref_last[b, h] = o[0]
    assert len({tuple(s) for s in seen}) > 3
    assert np.abs(state.double().cpu().numpy() - ref_state).max() <= 2.0 ** -18 * np.abs(ref_state).max()
