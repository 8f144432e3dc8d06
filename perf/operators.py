"""Linear attention with a decay for each head, and beam search over recurrent states: what is measured of them.

A case is one call of a public entry point (a training step: one forward and one backward call) on device tensors
that are already in place.  With `own` the library's entry points are called; without it the same operators are
computed from elementary tensor operations.

    decay     S_t = g_h S_{t-1} + k_t v_t^T,  o_t = scale S_t^T q_t,  g_h = exp(log_decay[h]),  from a given state or none
    train     the forward call, and the gradients of sum(o dO) + sum(S_n dS_n)
    step      one token of the same recurrence; with `parent` row b continues the state of row parent[b]
    select    of the candidates score_j + log softmax(logits_j)_t the n best of a batch entry's n beams
    reorder   the states of the beams follow their parents, in place
"""
import math

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def _attention(name, kind, B, H, L, dk, dv, dtype, **more):
    c = {"kind": kind, "B": B, "H": H, "L": L, "dk": dk, "dv": dv, "dtype": dtype, "layout": "bhld", "ragged": False, "carried": False}
    c.update(more)
    return {"name": name, **c} if name else c


def _step(name, B, H, dk, dv, dtype, n):
    c = {"kind": "step", "B": B, "H": H, "dk": dk, "dv": dv, "dtype": dtype, "n": n}
    return {"name": name, **c} if name else c


def _select(name, B, n, V, dtype, keep_slots):
    c = {"kind": "select", "B": B, "n": n, "V": V, "dtype": dtype, "keep_slots": keep_slots}
    return {"name": name, **c} if name else c


def _reorder(name, B, n, H, m, dv, layers):
    c = {"kind": "reorder", "B": B, "n": n, "H": H, "m": m, "dv": dv, "layers": layers}
    return {"name": name, **c} if name else c


def listed():
    return [
        # Prefill of one user's prompt: few heads, a length of no round number, the state kept for decoding.
        _attention("prompt_bf16", "decay", 1, 16, 777, 128, 128, "bf16"),
        # Decoder prefill of a batch: the largest call.
        _attention("prefill_bf16", "decay", 4, 16, 8192, 128, 128, "bf16"),
        # A padded batch of prompts at full precision that continue earlier states.
        _attention("padded_f32", "decay", 3, 12, 509, 64, 64, "f32", ragged=True, carried=True),
        # Queries and keys that are 256 features wide (a feature map's output), as a projection lays them out.
        _attention("features_bf16", "decay", 2, 12, 2048, 256, 64, "bf16", layout="blhd"),
        # Fine-tuning step of a decoder layer: forward and backward.
        _attention("train_bf16", "train", 2, 12, 4096, 64, 64, "bf16"),
        # A small training step at full precision, a ragged segment of longer texts: states come in and gradients leave.
        _attention("train_f32", "train", 1, 8, 1000, 64, 64, "f32", carried=True),
        # One decoded token for one user: latency.
        _step("step_one", 1, 16, 128, 128, "bf16", 1),
        # One decoded token for a serving batch of 16 users with 4 beams each; the beams' states follow their parents.
        _step("step_beams", 64, 32, 128, 128, "bf16", 4),
        # Beam search of one user.
        _select("select_one", 1, 4, 32000, "f32", False),
        # Beam search of a serving batch over a large vocabulary of odd size; surviving beams keep their slots.
        _select("select_batch", 32, 8, 131071, "bf16", True),
        # The states of one layer of one user's beams.
        _reorder("reorder_one", 1, 4, 12, 64, 64, 1),
        # The states of two decoder layers of a serving batch.
        _reorder("reorder_batch", 8, 4, 16, 256, 128, 2),
    ]


_WIDTHS = {  # (dk, dv): ordinary heads, features, and sizes that fill no tile
    "bf16": ((64, 64), (128, 128), (256, 64), (64, 128), (96, 80), (33, 65)),
    "f32": ((64, 64), (128, 128), (64, 128), (48, 56), (31, 33)),
}


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(("decay", "decay", "decay", "train", "train", "step", "select", "reorder"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind in ("decay", "train"):
        dk, dv = rng.choice(_WIDTHS[dtype])
        B, H = rng.choice((1, 1, 2, 3, 4, 6, 8)), rng.choice((1, 2, 4, 6, 8, 12, 16))
        # elements of q, k, v and out that the kind's largest listed case has for this type
        most = {("decay", "bf16"): 2.6e8, ("decay", "f32"): 9e6, ("train", "bf16"): 2.5e7, ("train", "f32"): 4e6}[kind, dtype]
        longest = max(2, int(most / (2 * B * H * (dk + dv))))
        return _attention(None, kind, B, H, _spread(rng, 1, min(longest, 65536)), dk, dv, dtype, layout=rng.choice(("bhld", "blhd")),
                          ragged=rng.random() < 0.3, carried=rng.random() < 0.5)
    if kind == "step":
        dk, dv = rng.choice(_WIDTHS[dtype])
        n = rng.choice((1, 2, 4, 5))
        H = rng.choice((1, 4, 12, 16, 32))
        return _step(None, n * _spread(rng, 1, 16 * 4 / n), H, dk, dv, dtype, n)
    if kind == "select":
        n = rng.choice((1, 2, 3, 4, 5, 8, 8))
        return _select(None, _spread(rng, 1, 32), n, _spread(rng, 1000, 131071), dtype, rng.random() < 0.5)
    return _reorder(None, _spread(rng, 1, 8), rng.choice((2, 3, 4, 4)), rng.choice((4, 8, 12, 16)), rng.choice((64, 128, 256)),
                    rng.choice((64, 64, 128)), rng.choice((1, 2)))


def _generator(seed, k=0):
    return torch.Generator(device="cuda").manual_seed(1000003 * seed + 7919 * k + 41)


def _log_decay(H):
    # memories of 2^5 to 2^11 tokens, one for each head
    e = torch.linspace(5.0, 11.0, H, dtype=torch.float64) if H > 1 else torch.tensor([7.0], dtype=torch.float64)
    return torch.log1p(-torch.exp2(-e)).float().cuda()


def _idempotent(parent):
    """Parents whose surviving beams stay where they are: [B, n]."""
    slots = torch.arange(parent.shape[1], device=parent.device).expand_as(parent)
    alive = torch.zeros_like(parent).scatter_(1, parent, 1).bool()
    return torch.where(alive, slots, parent)


def prepare(case, seed):
    g = _generator(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = {"case": case}
    if case["kind"] in ("decay", "train"):
        B, H, L, dk, dv = (case[k] for k in ("B", "H", "L", "dk", "dv"))
        dtype = _TORCH[case["dtype"]]

        def rows(d):
            return randn(*((B, H, L, d) if case["layout"] == "bhld" else (B, L, H, d))).to(dtype)

        s.update(Q=rows(dk), K=rows(dk), V=rows(dv), log_decay=_log_decay(H), lengths=None, state=None, dstate=None)
        if case["ragged"]:
            s["lengths"] = torch.randint(0, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            s["lengths"][-1] = L
        if case["carried"]:
            s["state"] = 4.0 * randn(B, H, dk, dv)
        if case["kind"] == "train":
            s["dOut"] = rows(dv)
            if case["carried"]:
                s["dstate"] = randn(B, H, dk, dv)
        return s
    if case["kind"] == "step":
        B, H, dk, dv = (case[k] for k in ("B", "H", "dk", "dv"))
        dtype = _TORCH[case["dtype"]]
        s.update(q=randn(B, H, dk).to(dtype), k=randn(B, H, dk).to(dtype), v=randn(B, H, dv).to(dtype), log_decay=_log_decay(H),
                 state=4.0 * randn(B, H, dk, dv), state_out=torch.zeros(B, H, dk, dv, device="cuda"), parent=None)
        if case["n"] > 1:   # beam b of a batch entry continues one of that entry's n beams
            own_beam = torch.randint(0, case["n"], (B,), generator=g, device="cuda")
            first = torch.arange(B, device="cuda") // case["n"] * case["n"]
            s["parent"] = (first + own_beam).to(torch.int32)
        return s
    if case["kind"] == "select":
        B, n, V = case["B"], case["n"], case["V"]
        logits = 3.0 * randn(B, n, V)
        logits[:, :, V - V // 500:] = float("-inf")   # entries of the output layer that stand for no token
        s["logits"] = logits.to(_TORCH[case["dtype"]])
        s["scores"] = torch.sort(-20.0 + randn(B, n), dim=1, descending=True).values.contiguous()
        s["finished"] = (torch.rand(B, n, generator=g, device="cuda") < 0.1).to(torch.uint8)
        s["eos"] = 2
        return s
    B, n, H, m, dv = (case[k] for k in ("B", "n", "H", "m", "dv"))
    # the recurrent state of a decoder layer: weighted values, their weights, and the exponents' shift
    s["states"] = [t for _ in range(case["layers"]) for t in (randn(B * n, H, m, dv), torch.rand(B * n, H, m, generator=g, device="cuda"),
                                                               randn(B * n, H))]
    s["parent"] = _idempotent(torch.randint(0, n, (B, n), generator=g, device="cuda")).to(torch.int32)
    return s


def run(state):
    case = state["case"]
    if own:
        return _run_own(case["kind"], state)
    return {"decay": _plain_decay, "train": _plain_train, "step": _plain_step, "select": _plain_select, "reorder": _plain_reorder}[case["kind"]](state)


def _run_own(kind, s):
    import paper_2603_04127_amd as dk

    if kind in ("decay", "train"):
        more = {"lengths": s["lengths"], "state": s["state"], "layout": s["case"]["layout"]}
        out, last = dk.dark_decay_fwd(s["Q"], s["K"], s["V"], s["log_decay"], want_state=True, **more)
        if kind == "decay":
            return out, last
        return out, last, dk.dark_decay_bwd(s["Q"], s["K"], s["V"], s["log_decay"], s["dOut"], dstate=s["dstate"], **more)
    if kind == "step":
        return dk.dark_decay_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"], parent=s["parent"], state_out=s["state_out"]), s["state_out"]
    if kind == "select":
        return dk.dark_beam_select(s["logits"], s["scores"], finished=s["finished"], eos=s["eos"], keep_slots=s["case"]["keep_slots"])
    dk.dark_state_reorder(s["states"], s["parent"])
    return s["states"]


# ---------------------------------------------------------------------------
# plain forms: chunk by chunk in 32 bits
# ---------------------------------------------------------------------------
_CHUNK = 128


def _heads_first(x, layout):
    return (x if layout == "bhld" else x.transpose(1, 2)).float()


def _back(x, case):
    x = x.to(_TORCH[case["dtype"]])
    return x.contiguous() if case["layout"] == "bhld" else x.transpose(1, 2).contiguous()


def _plain_scan(x1, x2, x3, a, lengths, S, offset, reverse):
    """y_t = sum over the rows c up to t of g^(t-c) (x1_t . x2_c) x3_c + g^(t+1-offset) S^T x1_t, and the state after the last row:
    g^n S + sum of g^(n-1-c+offset) x2_c x3_c^T.  `reverse`: rows counted from the sequence's end."""
    B, H, L, _ = x1.shape
    n = torch.full((B,), L, device=x1.device) if lengths is None else lengths.long()
    if reverse:   # rows n-1, n-2, ..., 0, and after them those behind the sequence
        t = torch.arange(L, device=x1.device)[None, :]
        order = torch.where(t < n[:, None], n[:, None] - 1 - t, t)[:, None, :, None]
        x1, x2, x3 = (torch.gather(x, 2, order.expand(-1, H, -1, x.shape[3])) for x in (x1, x2, x3))
    a = a.view(1, H, 1, 1)
    y = []
    for c0 in range(0, L, _CHUNK):
        q, k, v = (x[:, :, c0:c0 + _CHUNK] for x in (x1, x2, x3))
        r = torch.arange(q.shape[2], device=q.device)
        rows = (n - c0).clamp(0, q.shape[2]).view(B, 1, 1, 1)
        there = r.view(1, 1, -1, 1) < rows
        k, v = torch.where(there, k, 0.0), torch.where(there, v, 0.0)
        apart = r[:, None] - r[None, :]
        weight = torch.where(apart >= 0, torch.exp(a * apart.clamp(min=0)), 0.0)
        o = torch.matmul(torch.matmul(q, k.transpose(2, 3)) * weight, v) + torch.exp(a * (r.view(1, 1, -1, 1) + 1 - offset)) * torch.matmul(q, S)
        y.append(torch.where(there, o, 0.0))
        left = torch.where(there, torch.exp(a * (rows - 1 - r.view(1, 1, -1, 1) + offset).clamp(min=0)), 0.0)
        S = torch.exp(a * rows) * S + torch.matmul((k * left).transpose(2, 3), v)
    y = torch.cat(y, 2)
    return (torch.gather(y, 2, order.expand(-1, H, -1, y.shape[3])) if reverse else y), S


def _plain_decay(s):
    case = s["case"]
    q, k, v = (_heads_first(s[x], case["layout"]) for x in "QKV")
    first = torch.zeros(*q.shape[:2], q.shape[3], v.shape[3], device=q.device) if s["state"] is None else s["state"]
    out, last = _plain_scan(q * case["dk"] ** -0.5, k, v, s["log_decay"], s["lengths"], first, 0, False)
    return _back(out, case), last


def _plain_train(s):
    case, a = s["case"], s["log_decay"]
    out, last = _plain_decay(s)
    q, k, v, do = (_heads_first(s[x], case["layout"]) for x in ("Q", "K", "V", "dOut"))
    do = do * case["dk"] ** -0.5
    zero = torch.zeros(*q.shape[:2], q.shape[3], v.shape[3], device=q.device)
    first = zero if s["state"] is None else s["state"]
    dlast = zero if s["dstate"] is None else s["dstate"]
    dq, _ = _plain_scan(do, v, k, a, s["lengths"], first.transpose(2, 3), 0, False)
    dv, dfirst = _plain_scan(k, q, do, a, s["lengths"], dlast, 1, True)
    dkey, _ = _plain_scan(v, do, q, a, s["lengths"], dlast.transpose(2, 3), 1, True)
    grads = {"dQ": _back(dq, case), "dK": _back(dkey, case), "dV": _back(dv, case)}
    if s["state"] is not None:
        grads["dstate"] = dfirst
    return out, last, grads


def _plain_step(s):
    S = s["state"] if s["parent"] is None else s["state"][s["parent"].long()]
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    S = torch.exp(s["log_decay"])[None, :, None, None] * S + k[..., None] * v[..., None, :]
    out = (q[..., None] * S).sum(2) * q.shape[-1] ** -0.5
    s["state_out"].copy_(S)
    return out.to(s["v"].dtype), s["state_out"]


def _plain_select(s):
    logits, scores = s["logits"].double(), s["scores"].double()   # candidates of two beams can lie close together
    B, n, V = logits.shape
    top = logits.amax(2, keepdim=True)
    total = top + torch.log(torch.exp(logits - top).sum(2, keepdim=True))
    cand = scores[:, :, None] + logits - total
    kept = torch.full_like(cand, float("-inf"))
    kept[:, :, s["eos"]] = scores
    cand = torch.where(s["finished"].bool()[:, :, None], kept, cand)
    # the stable sort leaves equal candidates in the order of their index; a beam has at most n of the n best
    value, token = torch.sort(cand, dim=2, descending=True, stable=True)
    value, token = value[:, :, :n].reshape(B, n * n), token[:, :, :n].reshape(B, n * n)
    value, at = torch.sort(value, dim=1, descending=True, stable=True)
    value, at = value[:, :n], at[:, :n]
    parent, token = at // n, torch.gather(token, 1, at)
    if s["case"]["keep_slots"]:
        slots = torch.arange(n, device=at.device)
        again = ((parent[:, :, None] == parent[:, None, :]) & (slots[None, :] < slots[:, None])).any(2)   # its beam came before
        alive = torch.zeros_like(parent).scatter_(1, parent, 1)
        free = torch.sort(alive, dim=1, stable=True).indices
        slot = torch.where(again, torch.gather(free, 1, (torch.cumsum(again, 1) - 1).clamp(min=0)), parent)
        value, parent, token = (torch.zeros_like(x).scatter_(1, slot, x) for x in (value, parent, token))
    return value.float(), parent.to(torch.int32), token.to(torch.int32)


def _plain_reorder(s):
    B, n = s["parent"].shape
    rows = (s["parent"].long() + n * torch.arange(B, device=s["parent"].device)[:, None]).reshape(-1)
    for t in s["states"]:
        t.copy_(t[rows])
    return s["states"]


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _sequence(q, k, v, a, n, first, do=None, dlast=None):
    """One (batch entry, head): every weight g^(t-l) of the n rows written out, a block of rows at a time."""
    L, scale = q.shape[0], q.shape[1] ** -0.5
    out, last = torch.zeros_like(v), math.exp(a * n) * first
    dq, dkey, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    t = torch.arange(n, device=q.device, dtype=torch.float64)
    q, k, v = q[:n], k[:n], v[:n]
    last = last + (k * torch.exp(a * (n - 1 - t))[:, None]).T @ v
    decayed = torch.exp(a * (t + 1))[:, None]
    out[:n] = scale * decayed * (q @ first)
    if do is not None:
        do = do[:n]
        dq[:n] = scale * decayed * (do @ first.T)
        left = torch.exp(a * (n - 1 - t))[:, None]
        dkey[:n], dv[:n] = left * (v @ dlast.T), left * (k @ dlast)
        dfirst = math.exp(a * n) * dlast + scale * (q * decayed).T @ do
    for r0 in range(0, n, 1024):
        r1 = min(n, r0 + 1024)
        apart = t[r0:r1, None] - t[None, :r1]
        weight = scale * torch.where(apart >= 0, torch.exp(a * apart.clamp(min=0)), torch.zeros((), dtype=torch.float64, device=q.device))
        P = weight * (q[r0:r1] @ k[:r1].T)
        out[r0:r1] += P @ v[:r1]
        if do is not None:
            R = weight * (do[r0:r1] @ v[:r1].T)
            dq[r0:r1] += R @ k[:r1]
            dkey[:r1] += R.T @ q[r0:r1]
            dv[:r1] += P.T @ do[r0:r1]
    return (out, last) if do is None else (out, last, dq, dkey, dv, dfirst)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("decay", "train"):
        B, H, L, dk, dv = (case[k] for k in ("B", "H", "L", "dk", "dv"))
        first = lambda x: (x if case["layout"] == "bhld" else x.transpose(1, 2)).double()
        back = lambda x: (x if case["layout"] == "bhld" else x.transpose(1, 2)).contiguous()
        names = ["Q", "K", "V"] + (["dOut"] if kind == "train" else [])
        x = {k: first(s[k]) for k in names}
        zero = torch.zeros(dk, dv, dtype=torch.float64, device="cuda")
        a = s["log_decay"].double().tolist()
        n = [L] * B if s["lengths"] is None else s["lengths"].tolist()
        heads = []
        for b in range(B):
            for h in range(H):
                S = zero if s["state"] is None else s["state"][b, h].double()
                dS = zero if s["dstate"] is None else s["dstate"][b, h].double()
                heads.append(_sequence(x["Q"][b, h], x["K"][b, h], x["V"][b, h], a[h], n[b], S,
                                       *((x["dOut"][b, h], dS) if kind == "train" else ())))
        whole = [torch.stack([hd[i] for hd in heads]).unflatten(0, (B, H)) for i in range(len(heads[0]))]
        if kind == "decay":
            return back(whole[0]), whole[1]
        grads = {"dQ": back(whole[2]), "dK": back(whole[3]), "dV": back(whole[4])}
        if s["state"] is not None:
            grads["dstate"] = whole[5]
        return back(whole[0]), whole[1], grads
    if kind == "step":
        B, H, dk, dv = (case[k] for k in ("B", "H", "dk", "dv"))
        rows = range(B) if s["parent"] is None else s["parent"].tolist()
        g = torch.exp(s["log_decay"].double())[:, None, None]
        S = torch.stack([g * s["state"][r].double() + torch.einsum("hi,hj->hij", s["k"][b].double(), s["v"][b].double()) for b, r in enumerate(rows)])
        out = torch.stack([torch.einsum("hi,hij->hj", s["q"][b].double(), S[b]) for b in range(B)]) / math.sqrt(dk)
        return out, S
    if kind == "select":
        return _exact_select(case, s)
    n = case["n"]
    rows = [b * n + p for b, of in enumerate(s["parent"].tolist()) for p in of]
    return [torch.stack([t[r] for r in rows]) for t in s["states"]]


def _exact_select(case, s):
    B, n, V = case["B"], case["n"], case["V"]
    scores, parents, tokens = [], [], []
    for b in range(B):
        cand = []   # (value, beam, token)
        for j in range(n):
            score = float(s["scores"][b, j])
            if int(s["finished"][b, j]):
                cand.append((score, j, s["eos"]))
                continue
            row = s["logits"][b, j].double()
            logp = score + torch.log_softmax(row, 0).cpu()
            edge = float(torch.topk(logp, min(n, V)).values[-1])
            cand += [(float(logp[t]), j, t) for t in torch.nonzero(logp >= edge)[:, 0].tolist()]
        best = sorted(cand, key=lambda c: (-c[0], c[1], c[2]))[:n]
        if case["keep_slots"]:
            slots = [None] * n
            rest = []
            for c in best:
                if slots[c[1]] is None:
                    slots[c[1]] = c
                else:
                    rest.append(c)
            best = [c if c is not None else rest.pop(0) for c in slots]
        scores.append([c[0] for c in best])
        parents.append([c[1] for c in best])
        tokens.append([c[2] for c in best])
    return (torch.tensor(scores, dtype=torch.float64), torch.tensor(parents, dtype=torch.int32), torch.tensor(tokens, dtype=torch.int32))


def work(case):
    kind = case["kind"]
    if kind in ("decay", "train"):
        B, H, L, dk, dv = (case[k] for k in ("B", "H", "L", "dk", "dv"))
        n, size = B * H * L, 4 if case["dtype"] == "f32" else 2
        states = 4 * B * H * dk * dv * (2 if case["carried"] else 1)
        # forward: the state is updated and read once for each token
        moved, flops = n * 2 * (dk + dv) * size + states, n * 4 * dk * dv
        if kind == "train":   # the forward state again, the backward one, and three readouts
            moved += n * (4 * dk + 3 * dv) * size + (3 * 4 * B * H * dk * dv if case["carried"] else 0)
            flops += n * 10 * dk * dv
        return {"bytes": moved, "flops": flops}
    if kind == "step":
        B, H, dk, dv = (case[k] for k in ("B", "H", "dk", "dv"))
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": B * H * (8 * dk * dv + 2 * (dk + dv) * size), "flops": B * H * 5 * dk * dv}
    if kind == "select":
        rows = case["B"] * case["n"]
        return {"bytes": rows * case["V"] * (4 if case["dtype"] == "f32" else 2) + rows * 17, "flops": rows * case["V"] * 4}
    B, n, H, m, dv = (case[k] for k in ("B", "n", "H", "m", "dv"))
    # on average n (1 - 1/n)^n of n drawn parents' beams are dropped: that many rows are read and written
    moved = B * n * (1.0 - 1.0 / n) ** n
    return {"bytes": case["layers"] * moved * 2 * 4 * H * (m * dv + m + 1), "flops": 0}
