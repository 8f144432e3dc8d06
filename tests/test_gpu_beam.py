"""Beam search over recurrent states: selection against the fp64 oracle, states that follow their beams, and both with decoding."""
import numpy as np
import pytest
import torch

import paper_2603_04127_amd as dk
from oracle import decay_oracle as D

pytestmark = pytest.mark.gpu
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def _check(logits, scores, finished=None, eos=0):
    for keep in (False, True):
        s, p, t = dk.dark_beam_select(logits.cuda(), scores.cuda(), finished=None if finished is None else finished.cuda(), eos=eos, keep_slots=keep)
        s, p, t = s.cpu().numpy(), p.cpu().numpy(), t.cpu().numpy()
        for b in range(logits.shape[0]):
            ws, wp, wt = D.beam_select(logits[b].float().numpy(), scores[b].numpy(), None if finished is None else finished[b].numpy(), eos, keep)
            assert p[b].tolist() == wp and t[b].tolist() == wt, (b, keep, p[b], wp, t[b], wt)
            # the score is rounded once to fp32; the sum of exponentials (fp32 terms of 2^-22) moves its logarithm by 2^-22
            with np.errstate(invalid="ignore"):   # -inf beside -inf
                assert np.all((s[b] == ws) | (np.abs(s[b] - ws) <= 2.0 ** -24 * np.abs(ws) + 2.0 ** -21)), (b, s[b], ws)


def _problem(seed, B, n, V, dtype):
    g = torch.Generator().manual_seed(seed)
    return (3 * torch.randn(B, n, V, generator=g)).to(TORCH[dtype]), -20 + torch.randn(B, n, generator=g)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1), (2, 4, 2), (3, 4, 7), (1, 4, 32000), (2, 8, 50001), (5, 3, 1000), (1, 32, 2049), (2, 17, 999), (64, 8, 8193), (1, 2, 1000003)])
def test_selection(shape, dtype):
    logits, scores = _problem(sum(shape), *shape, dtype)
    _check(logits, scores)
    scores[:, 1:] = float("-inf")   # the first step: one beam in use
    _check(logits, scores)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 32, 50001), (1, 32, 131071)])
def test_lists_too_long_to_be_staged(shape, dtype):
    # n n entries a slice: more than the second kernel brings to LDS, so that it reads them where they are
    logits, scores = _problem(sum(shape), *shape, dtype)
    logits[:, 3, 100:] = float("-inf")   # slices without an entry
    logits[:, 4, ::7] = float("nan")
    finished = torch.arange(shape[1]).repeat(shape[0], 1) % 5 == 2
    _check(logits, scores, finished, 7)
    scores[:, 1:] = float("-inf")
    _check(logits, scores)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_candidates(dtype):
    logits, scores = _problem(1, 3, 4, 3000, dtype)
    logits = logits.round()          # many equal logits in a row
    logits[1] = logits[1, :1]        # equal beams
    scores[1] = -3.0
    logits[2] = 0.0                  # everything equal
    scores[2] = 0.0
    _check(logits, scores)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_rows(dtype):
    inf, nan = float("inf"), float("nan")
    logits, scores = _problem(2, 6, 4, 2500, dtype)
    logits[0, 0] = -inf                              # a row without a token
    logits[1] = -inf                                 # no row has any
    logits[1, 2, [5, 2000]] = torch.tensor([1.0, 2.0], dtype=logits.dtype)   # two candidates for four places
    logits[2, :, ::2] = nan
    logits[3, 1, 77] = inf
    logits[4] = -inf
    scores[5] = torch.tensor([nan, -inf, inf, -5.0])
    _check(logits, scores)
    logits, scores = _problem(3, 1, 4, 100, dtype)
    logits = torch.where(logits < 0, torch.finfo(logits.dtype).min, logits)   # masked by the type's lowest value
    _check(logits, scores)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [301, 20001])
def test_infinities_and_nan_beside_numbers(V, dtype):
    logits, scores = _problem(10, 6, 4, V, dtype)
    inf = float("inf")
    bits = logits.view(torch.int16 if dtype == "bf16" else torch.int32)
    bits[0, :, 1::3] = 0x7F81 if dtype == "bf16" else 0x7F800001   # signalling NaN in each half of a word, at every lane
    logits[1, :, 0::2] = -inf
    logits[2, :, 1::2] = -inf
    logits[3] = -3.0 + 0.01 * logits[3]              # below zero, and close together
    logits[4, 0, 5], logits[4, 1, 6], logits[4, 2] = inf, inf, -inf
    logits[4, 2, [8, 9]] = torch.tensor([inf, 1.0], dtype=logits.dtype)
    logits[4, 3, :] = -inf
    logits[4, 3, V - 1] = -0.0
    logits[5] = torch.where(logits[5] > 0, 0.0, -0.0)   # both zeros
    _check(logits, scores)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 20000])
def test_logits_near_the_end_of_the_type(V, dtype):
    logits, scores = _problem(9, 4, 4, V, dtype)
    low, high = torch.finfo(logits.dtype).min, torch.finfo(logits.dtype).max
    logits[0, 1] = low               # a row masked as a whole: every token has the same share
    logits[1] = low
    logits[1, 2, 17] = low / 2
    logits[2, 0, [3, V - 1]] = high  # two tokens share everything, the others end below the range: -infinity, or nearly
    logits[3] *= 2.0 ** 20           # large, but not so large that log2 e is too much
    _check(logits, scores)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", [torch.uint8, torch.bool])
def test_finished_beams(kind, dtype):
    logits, scores = _problem(4, 4, 4, 1500, dtype)
    scores[:, 0] = -8.0
    finished = torch.tensor([[1, 0, 0, 0], [0, 1, 0, 1], [1, 1, 1, 1], [1, 0, 1, 0]]).to(kind)
    scores[3, 1] = float("-inf")     # dead, finished and alive ones together
    logits[3, 0] = float("nan")      # not read
    for eos in (0, 2, 1499):
        _check(logits, scores, finished, eos)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,kind", [((1, 17, 999), "tiny"), ((3, 17, 999), "tiny"), ((1, 4, 999), "tiny"), ((1, 32, 73000), "rising"), ((2, 32, 999), "same"),
                                        ((1, 32, 73000), "huge"), ((2, 5, 20001), "huge")])
def test_candidates_that_no_double_tells_apart(shape, kind, dtype):
    # all winners are beam 0's largest logits, equal ones by the lowest token, though many values are one and the same double
    B, n, V = shape
    row = torch.linspace(-3, 3, V)[torch.randperm(V, generator=torch.Generator().manual_seed(V))]
    if kind in ("tiny", "rising"):
        row = 1e-20 * torch.arange(V) if kind == "tiny" else torch.linspace(-3, 3, V)
    row = row.to(TORCH[dtype])
    scores = torch.full((n,), float("-inf"))
    scores[0] = -1e20
    if kind == "tiny":
        scores = -torch.arange(n, dtype=torch.float32)
    elif kind == "same":
        scores[:] = -1e20
    elif kind == "huge":
        scores[0], row[V // 2] = -2.0, 2.0 ** 100
    want = np.lexsort((np.arange(V), -row.double().numpy()))[:n]
    for keep in (False, True):
        room = [torch.full((3, B, n), 7, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)]
        s, p, t = dk.dark_beam_select(row.expand(B, n, V).contiguous().cuda(), scores.repeat(B, 1).cuda(), keep_slots=keep, out=[r[1] for r in room])
        assert (p == 0).all() and (t.cpu().numpy() == want).all(), (keep, p, t, want)
        x = row.double().numpy() - float(row.max())
        value = float(scores[0]) - np.log(np.exp(x).sum()) + x[want]
        # the score's rounding, and the sum's: at most 31 + 8 additions one after the other and an exponential off by 2^-23
        assert np.all(np.abs(s.cpu().numpy() - value) <= 2.0 ** -24 * np.abs(value) + 2.0 ** -18)
        assert all((r[0] == 7).all() and (r[2] == 7).all() for r in room)   # nothing beside the results


def _sums_error(rows):
    """How far the logarithms of the rows' sums of exponentials are off: [B, V] rows, each with a score that leaves its best candidate near
    zero, so that the rounding of the result hides nothing."""
    x = rows.double().numpy()
    top = x.max(1, keepdims=True)
    total = np.log(np.exp(x - top).sum(1))
    scores = torch.from_numpy(total).float()
    s, _, t = dk.dark_beam_select(rows[:, None].contiguous().cuda(), scores[:, None].contiguous().cuda())
    assert (x[np.arange(len(x)), t[:, 0].cpu().numpy()] == top[:, 0]).all()
    return np.abs(s[:, 0].double().cpu().numpy() - (scores.double().numpy() - total))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [8192, 24576])
def test_sums_of_equal_logits(V, dtype):
    # whole slices of equal terms: every addition by halves is exact, and an exponential is off by at most 2^-23
    value = torch.cat([torch.tensor([513.117, -0.5, 0.0, 1e-3, -1e5, 1e6]), 700 * torch.rand(250, generator=torch.Generator().manual_seed(V)) - 350])
    worst = _sums_error(value[:, None].expand(-1, V).to(TORCH[dtype])).max()
    assert worst <= 2.0 ** -23 * 1.01


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [False, True])
def test_sums_within_their_bound(bad, dtype):
    # the bound of dark.h: 14 additions, an exponential, and exponents of up to 2^5 whose roundings may all have one sign
    V, g = 131071, torch.Generator().manual_seed(8)
    rows = torch.stack([torch.zeros(V) - x for x in (2.1, 7.3, 9.77, 10.9, 11.3, 11.77)] + [s * torch.randn(V, generator=g) for s in (0.1, 1.0, 3.0, 10.0)])
    rows[:6, 5] = 0.0   # one large logit, and as much in all the others together
    rows = (rows + torch.linspace(-40, 40, 10)[:, None]).to(TORCH[dtype])
    error = _sums_error(rows if not bad else torch.where(torch.arange(V) % 301 == 7, float("-inf"), rows))
    if bad:   # NaN count for nothing, as -infinity does
        assert torch.equal(*(torch.stack(dk.dark_beam_select(torch.where(torch.arange(V) % 301 == 7, b, rows)[:, None].contiguous().cuda(),
                                                             torch.zeros(10, 1, device="cuda"))[:1]) for b in (float("-inf"), float("nan"))))
    print(error)
    assert error.max() <= 2.0 ** -19, error


def test_scores_in_place_and_given_outputs():
    logits, scores = _problem(5, 2, 4, 5000, "f32")
    logits, scores = logits.cuda(), scores.cuda()
    want = dk.dark_beam_select(logits, scores)
    parent, token = (torch.empty(2, 4, dtype=torch.int32, device="cuda") for _ in range(2))
    got = dk.dark_beam_select(logits, scores, out=(scores, parent, token))
    assert got[0] is scores and all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("n", [1, 2, 4, 5, 8, 13, 32])
@pytest.mark.parametrize("tail,dtype", [((12, 64, 64), torch.float32), ((7,), torch.float32), ((3, 5), torch.bfloat16), ((1, 1000), torch.uint8), ((16, 129), torch.float32)])
def test_reorder(n, tail, dtype):
    g = torch.Generator().manual_seed(n)
    B = 3
    states = [(100 * torch.randn(B * n, *tail, generator=g)).to(dtype).cuda(), torch.randn(B, n, 6, generator=g).cuda()]
    for kind in range(4):
        if kind == 0:
            parent = torch.stack([torch.randperm(n, generator=g) for _ in range(B)])            # cycles
        elif kind == 1:
            parent = torch.randint(0, n, (B, n), generator=g)                                    # the same index twice
        elif kind == 2:
            parent = torch.arange(n).repeat(B, 1)                                                # nothing moves
        else:
            parent = torch.randint(-2, n + 2, (B, n), generator=g)                               # some are no beams
        follow = torch.where((parent >= 0) & (parent < n), parent, torch.arange(n).repeat(B, 1)).cuda()
        want = [torch.stack([x.reshape(B, n, -1)[b][follow[b]] for b in range(B)]).reshape(x.shape) for x in states]
        dk.dark_state_reorder(states, parent.to(torch.int32).cuda())
        assert all(torch.equal(x, y) for x, y in zip(states, want)), kind


def test_reorder_many_tensors_and_none():
    parent = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    many = [torch.arange(2 * (i + 1), dtype=torch.float32, device="cuda").reshape(2, -1) for i in range(37)]
    want = [t.flip(0) for t in many]
    dk.dark_state_reorder(many, parent)
    assert all(torch.equal(x, y) for x, y in zip(many, want))
    dk.dark_state_reorder([], parent)
    dk.dark_state_reorder([torch.empty(2, 0, device="cuda")], parent)


def test_offsets_beyond_32_bits():
    B, n, V = 1081, 8, 249999
    g = torch.Generator(device="cuda").manual_seed(7)
    logits = torch.zeros(B, n, V, dtype=torch.bfloat16, device="cuda")
    assert logits.numel() > 1 << 31
    logits[-1] = torch.randn(n, V, generator=g, device="cuda")
    scores = -torch.rand(B, n, generator=g, device="cuda")
    s, p, t = dk.dark_beam_select(logits, scores)
    ws, wp, wt = dk.dark_beam_select(logits[-1:].clone(), scores[-1:].clone())   # smaller slices: sums of 2^-22 in another order
    assert torch.equal(p[-1:], wp) and torch.equal(t[-1:], wt) and ((s[-1:] - ws).abs() <= 2 * 2.0 ** -21 + 2.0 ** -23 * ws.abs()).all()
    assert (t[0] == torch.arange(n, device="cuda")).all() and (p[0] == scores[0].argmax()).all()   # equal logits: the best beam's first tokens
    states = torch.zeros(40, 4, 1 << 23, device="cuda")
    states[-1] = torch.randn(4, 1 << 23, generator=g, device="cuda")
    want = states[-1].clone()
    parent = torch.arange(4, dtype=torch.int32, device="cuda").repeat(40, 1)
    parent[-1] = torch.tensor([2, 2, 0, 1])
    dk.dark_state_reorder([states], parent)
    assert torch.equal(states[-1], want[parent[-1].long()]) and not states[0].any()


def _search(step, reorder, logits_of, B, n, V, steps, keep_slots):
    """Beam search with `step` (token features in, outputs back) and `reorder` (parents)."""
    scores = torch.full((B, n), float("-inf"))
    scores[:, 0] = 0.0
    finished = torch.zeros(B, n, dtype=torch.bool)
    token = torch.zeros(B, n, dtype=torch.int32)
    scores, finished, token = scores.cuda(), finished.cuda(), token.cuda()
    history = []
    for _ in range(steps):
        logits = logits_of(step(token)).reshape(B, n, V).contiguous()
        scores, parent, token = dk.dark_beam_select(logits, scores, finished=finished, eos=1, keep_slots=keep_slots)
        finished = torch.gather(finished, 1, parent.long()) | (token == 1)
        reorder(parent)
        history.append((parent.cpu(), token.cpu(), scores.cpu()))
    return history


@pytest.mark.parametrize("keep_slots", [False, True])
@pytest.mark.parametrize("fused", [False, True])
def test_beam_search_with_decayed_states(fused, keep_slots):
    # A prompt, then beam search over a toy model of one layer: the states as the library moves them against states that are
    # recomputed from each beam's own tokens.
    B, n, H, d, V, steps = 2, 4, 2, 64, 300, 12
    g = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    emb = [r(V, H, d) for _ in range(3)]
    head = r(H * d, V) * 0.2
    a = torch.tensor([-0.02, -0.3], device="cuda")
    prompt = [r(B, H, 37, d) for _ in range(3)]
    _, S = dk.dark_decay_fwd(*prompt, a, want_state=True)
    state = [S.repeat_interleave(n, 0).contiguous(), torch.empty(B * n, H, d, d, device="cuda")]
    pending = [None]

    def step(token):
        x = [e[token.reshape(-1).long()].contiguous() for e in emb]
        out = dk.dark_decay_step(*x, a, state[0], parent=pending[0], state_out=state[1])
        state.reverse()
        return out

    def reorder(parent):
        if fused:    # the next step reads its states through the parents
            pending[0] = (parent + n * torch.arange(B, dtype=torch.int32, device="cuda")[:, None]).reshape(-1).contiguous()
        else:
            dk.dark_state_reorder([state[0]], parent)

    history = _search(step, reorder, lambda out: out.reshape(B * n, -1) @ head, B, n, V, steps, keep_slots)
    # every beam's tokens, traced back through its parents
    for b in range(B):
        for j in range(n):
            at, tokens, done = j, [], []
            for parent, token, _ in reversed(history):
                tokens.append(int(token[b, at]))
                at = int(parent[b, at])
            tokens = tokens[::-1]
            score, x = 0.0, [0] + tokens[:-1]
            seq = [torch.cat([p[b], e[torch.tensor(x, device="cuda")].transpose(0, 1)], 1).double().cpu().numpy() for p, e in zip(prompt, emb)]
            out = np.stack([D.forward(seq[0][h], seq[1][h], seq[2][h], float(a[h]), np.zeros((d, d)), d ** -0.5)[0][37:] for h in range(H)], 1)
            logp = torch.log_softmax(torch.from_numpy(out.reshape(steps, -1)) @ head.double().cpu(), 1)
            for t in range(steps):
                score += float(logp[t, tokens[t]])
                if tokens[t] == 1:
                    break
            # 12 sums of log-probabilities from fp32 products over 128 terms
            assert abs(score - float(history[-1][2][b, j])) <= 1e-3, (b, j, score, history[-1][2][b])


def test_reorder_the_states_of_the_feature_map_s_decoding():
    # states of dark_decode_step follow their beams: the same as decoding each beam's own tokens from the start
    B, n, H, d, m, steps = 1, 3, 2, 64, 128, 6
    g = torch.Generator(device="cuda").manual_seed(6)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda") * 0.5
    W = torch.randn(H, m, d, generator=g, device="cuda")
    state = dk.decode_state(B * n, H, m, d)
    tokens = [[r(B * n, H, d) for _ in range(3)] for _ in range(steps)]
    lineage = [[] for _ in range(n)]
    parents = [[0, 1, 2], [2, 0, 0], [1, 2, 1], [0, 0, 0], [2, 1, 0], [0, 1, 2]]
    for t in range(steps):
        out = dk.dark_decode_step(*tokens[t], None, W, state)
        lineage = [x + [(t, j)] for j, x in enumerate(lineage)]
        dk.dark_state_reorder(list(state), torch.tensor([parents[t]], dtype=torch.int32, device="cuda"))
        lineage = [lineage[p] for p in parents[t]]
    for j in range(n):
        alone = dk.decode_state(1, H, m, d)
        for t, at in lineage[j]:
            dk.dark_decode_step(*(x[at:at + 1].contiguous() for x in tokens[t]), None, W, alone)
        assert all(torch.allclose(x[j:j + 1], y, rtol=1e-5, atol=1e-6) for x, y in zip(state, alone))


def test_captured_selection_replays():
    logits, scores = (t.cuda() for t in _problem(7, 4, 4, 20000, "bf16"))
    states = [torch.randn(16, 4, 64, device="cuda")]

    def work():
        out = dk.dark_beam_select(logits, scores)
        dk.dark_state_reorder(states, out[1])
        return out

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for _ in range(3):
        logits.copy_(3 * torch.randn_like(logits))
        first = states[0].clone()
        graph.replay()
        torch.cuda.synchronize()
        got, moved = [t.clone() for t in held], states[0].clone()
        states[0].copy_(first)
        assert all(torch.equal(x, y) for x, y in zip(got, work())) and torch.equal(states[0], moved)
