"""The gated delta rule (linear attention whose state corrects itself), and the drawing of tokens from logits: what is measured of them.

A case is one call of a public entry point (a training step: one forward and one backward call) on device tensors
that are already in place.  With `own` the library's entry points are called; without it the same operators are
computed from elementary tensor operations.

    delta     S_t = a_t S_{t-1} + k_t u_t^T,  u_t = beta_t (v_t - a_t S_{t-1}^T k_t),  o_t = scale S_t^T q_t,  a_t = exp(log_gate_t)
    train     the forward call, and the gradients of sum(o dO) + sum(S_n dS_n)
    step      one token of the same recurrence; with `parent` row b continues the state of row parent[b]
    sample    a token of each row, from softmax(logits / temperature) restricted to the top_k likeliest, to the likeliest that hold
              top_p of their sum, and to those of min_p times the likeliest's probability; by a given random number
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


def _sample(name, B, V, dtype, mix):
    c = {"kind": "sample", "B": B, "V": V, "dtype": dtype, "mix": mix}
    return {"name": name, **c} if name else c


def listed():
    return [
        # Prefill of one user's prompt: few heads, a length of no round number, the state kept for decoding.
        _attention("prompt_bf16", "delta", 1, 16, 777, 128, 128, "bf16"),
        # Decoder prefill of a batch: the largest call.
        _attention("prefill_bf16", "delta", 4, 16, 8192, 128, 128, "bf16"),
        # Values twice as wide as the keys, as a projection lays them out (heads behind the rows).
        _attention("wide_bf16", "delta", 2, 8, 2048, 128, 256, "bf16", layout="blhd"),
        # A padded batch of prompts at full precision that continue earlier states.
        _attention("padded_f32", "delta", 3, 12, 509, 64, 64, "f32", ragged=True, carried=True),
        # Fine-tuning step of a decoder layer: forward and backward.
        _attention("train_bf16", "train", 2, 12, 4096, 64, 64, "bf16"),
        # The same for a padded batch of wider heads that continues earlier segments: states come in and gradients leave.
        _attention("train_padded_bf16", "train", 3, 8, 1533, 128, 128, "bf16", layout="blhd", ragged=True, carried=True),
        # A small training step at full precision.
        _attention("train_f32", "train", 1, 8, 1000, 64, 64, "f32"),
        # One decoded token for one user: latency.
        _step("step_one", 1, 16, 128, 128, "bf16", 1),
        # One decoded token for a serving batch of 16 users with 4 beams each; the beams' states follow their parents.
        _step("step_beams", 64, 32, 128, 128, "bf16", 4),
        # The next token of one user: top_k, top_p and min_p together.
        _sample("sample_one", 1, 32000, "f32", "all"),
        # A serving batch over a large vocabulary of odd size; every user has settings of their own, the greedy and the unrestricted among them.
        _sample("sample_batch", 256, 131071, "bf16", "mixed"),
        # Rollouts for training: nothing is restricted.
        _sample("sample_rollout", 64, 65537, "f32", "none"),
    ]


_WIDTHS = {  # (dk, dv): ordinary heads, wide values and keys, and sizes that fill no tile
    "bf16": ((64, 64), (128, 128), (128, 256), (64, 128), (256, 128), (96, 80), (33, 65)),
    "f32": ((64, 64), (128, 128), (64, 128), (48, 56), (31, 33)),
}


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(("delta", "delta", "delta", "train", "train", "step", "sample", "sample"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind in ("delta", "train"):
        dk, dv = rng.choice(_WIDTHS[dtype])
        B, H = rng.choice((1, 1, 2, 3, 4, 6, 8)), rng.choice((1, 2, 4, 6, 8, 12, 16))
        # elements of q, k, v and out that the kind's largest listed case has for this type
        most = {("delta", "bf16"): 2.6e8, ("delta", "f32"): 9e6, ("train", "bf16"): 1.8e7, ("train", "f32"): 2e6}[kind, dtype]
        longest = max(2, int(most / (2 * B * H * (dk + dv))))
        return _attention(None, kind, B, H, _spread(rng, 1, min(longest, 32768)), dk, dv, dtype, layout=rng.choice(("bhld", "blhd")),
                          ragged=rng.random() < 0.3, carried=rng.random() < 0.5)
    if kind == "step":
        dk, dv = rng.choice(_WIDTHS[dtype])
        n = rng.choice((1, 2, 4, 5))
        H = rng.choice((1, 4, 12, 16, 32))
        return _step(None, n * _spread(rng, 1, 16 * 4 / n), H, dk, dv, dtype, n)
    return _sample(None, _spread(rng, 1, 128), _spread(rng, 1000, 131071), dtype, rng.choice(("all", "mixed", "mixed", "none")))


def _generator(seed, k=0):
    return torch.Generator(device="cuda").manual_seed(1000003 * seed + 7919 * k + 43)


def prepare(case, seed):
    g = _generator(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    def unit(x):   # keys and queries of the delta rule have length one
        return x / x.norm(dim=-1, keepdim=True)

    s = {"case": case}
    if case["kind"] in ("delta", "train", "step"):
        B, H, dk, dv = (case[k] for k in ("B", "H", "dk", "dv"))
        dtype = _TORCH[case["dtype"]]
        rows = (B, H) if case["kind"] == "step" else (B, H, case["L"]) if case["layout"] == "bhld" else (B, case["L"], H)
        # decays that forget half within 2^2 to 2^10 tokens, by the head, moved by the token
        e = torch.linspace(2.0, 10.0, H, device="cuda") if H > 1 else torch.full((1,), 6.0, device="cuda")
        rate = math.log(2.0) * torch.exp2(-e)
        rate = rate.view(1, H) if case["kind"] == "step" else rate.view(1, H, 1) if case["layout"] == "bhld" else rate.view(1, 1, H)
        q, k = ("q", "k") if case["kind"] == "step" else ("Q", "K")
        s[q], s[k] = unit(randn(*rows, dk)).to(dtype), unit(randn(*rows, dk)).to(dtype)
        s["v" if case["kind"] == "step" else "V"] = randn(*rows, dv).to(dtype)
        s["log_gate"] = (-rate * torch.exp(0.5 * randn(*rows))).contiguous()
        s["beta"] = torch.sigmoid(1.5 * randn(*rows))
    if case["kind"] in ("delta", "train"):
        s.update(lengths=None, state=None, dstate=None)
        if case["ragged"]:
            s["lengths"] = torch.randint(0, case["L"] + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            s["lengths"][-1] = case["L"]
        if case["carried"]:
            s["state"] = randn(B, H, dk, dv)
        if case["kind"] == "train":
            s["dOut"] = randn(*rows, dv).to(dtype)
            if case["carried"]:
                s["dstate"] = randn(B, H, dk, dv)
        return s
    if case["kind"] == "step":
        s.update(state=randn(B, H, dk, dv), state_out=torch.zeros(B, H, dk, dv, device="cuda"), parent=None)
        if case["n"] > 1:   # beam b of a batch entry continues one of that entry's n beams
            own_beam = torch.randint(0, case["n"], (B,), generator=g, device="cuda")
            first = torch.arange(B, device="cuda") // case["n"] * case["n"]
            s["parent"] = (first + own_beam).to(torch.int32)
        return s
    B, V = case["B"], case["V"]
    logits = 2.5 * randn(B, V)
    logits[:, V - V // 500:] = float("-inf")   # entries of the output layer that stand for no token
    s["logits"] = logits.to(_TORCH[case["dtype"]])
    s["uniform"] = rand(B)
    s["temperature"] = 0.6 + 0.6 * rand(B)
    s["top_k"] = torch.full((B,), 50, dtype=torch.int32, device="cuda")
    s["top_p"], s["min_p"] = 0.85 + 0.12 * rand(B), 0.1 * rand(B)
    if case["mix"] == "none":
        s["top_k"].zero_(), s["top_p"].fill_(1.0), s["min_p"].zero_()
    if case["mix"] == "mixed":
        s["temperature"][rand(B) < 0.1] = 0.0
        s["top_k"] = torch.where(rand(B) < 0.5, 0, torch.randint(1, 400, (B,), generator=g, device="cuda")).to(torch.int32)
        s["top_p"][rand(B) < 0.3] = 1.0
        s["min_p"][rand(B) < 0.5] = 0.0
    return s


def run(state):
    kind = state["case"]["kind"]
    if own:
        return _run_own(kind, state)
    return {"delta": _plain_delta, "train": _plain_train, "step": _plain_step, "sample": _plain_sample}[kind](state)


def _run_own(kind, s):
    import paper_2603_04127_amd as dk

    if kind in ("delta", "train"):
        more = {"lengths": s["lengths"], "state": s["state"], "layout": s["case"]["layout"]}
        out, last = dk.dark_delta_fwd(s["Q"], s["K"], s["V"], s["log_gate"], s["beta"], want_state=True, **more)
        if kind == "delta":
            return out, last
        return out, last, dk.dark_delta_bwd(s["Q"], s["K"], s["V"], s["log_gate"], s["beta"], s["dOut"], dstate=s["dstate"], **more)
    if kind == "step":
        return dk.dark_delta_step(s["q"], s["k"], s["v"], s["log_gate"], s["beta"], s["state"], parent=s["parent"], state_out=s["state_out"]), s["state_out"]
    return dk.dark_sample(s["logits"], s["uniform"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                          want_logprob=True)


# ---------------------------------------------------------------------------
# plain forms: chunk by chunk in 32 bits
# ---------------------------------------------------------------------------
_CHUNK = 64


class _Chunks:
    """A call's operands as [B, H, chunks, 64, ..] in 32 bits, zero (no key, no gate) behind a sequence, and what a chunk needs of itself:

    G the sum of its log gates up to a row, D_ti = exp(G_t - G_i) for i <= t, E the same below the diagonal times k_t . k_i,
    T = (I + diag(beta) E)^-1."""

    def __init__(self, s, names):
        case = s["case"]
        B, H, L = (case[k] for k in ("B", "H", "L"))
        self.case, self.C, self.n = case, min(_CHUNK, L), -(-L // min(_CHUNK, L))
        pad = self.n * self.C - L
        length = torch.full((B,), L, device="cuda") if s["lengths"] is None else s["lengths"].long()
        there = (torch.arange(L, device="cuda")[None] < length[:, None])[:, None, :, None]

        def chunks(x):
            x = x if x.dim() == 4 else x[..., None]
            x = torch.where(there, (x if case["layout"] == "bhld" else x.transpose(1, 2)).float(), 0.0)
            return torch.nn.functional.pad(x, (0, 0, 0, pad)).view(B, H, self.n, self.C, -1)

        self.there = there
        for name in names:
            setattr(self, name, chunks(s[name]))
        G = torch.cumsum(chunks(s["log_gate"]).double(), 3)
        self.beta, self.gamma, self.Gamma = chunks(s["beta"]), torch.exp(G).float(), torch.exp(G[:, :, :, -1:]).float()
        self.left = torch.exp(G[:, :, :, -1:] - G).float()
        r = torch.arange(self.C, device="cuda")
        lower = r[:, None] >= r[None, :]
        self.D = torch.where(lower, torch.exp((G - G.transpose(3, 4)).masked_fill(~lower, 0.0)), 0.0).float()
        self.KK = torch.matmul(self.K, self.K.transpose(3, 4))
        self.E = (self.D * self.KK).masked_fill(r[:, None] <= r[None, :], 0.0)
        A = self.beta * self.E
        self.T = torch.eye(self.C, device="cuda").expand_as(A).clone()
        for i in range(1, self.C):   # row after row
            self.T[..., i, :i] = -torch.matmul(A[..., i:i + 1, :i], self.T[..., :i, :i])[..., 0, :]
        self.scale = case["dk"] ** -0.5

    def back(self, x, dtype):
        B, H, L = (self.case[k] for k in ("B", "H", "L"))
        x = torch.where(self.there, x.reshape(B, H, self.n * self.C, -1)[:, :, :L], 0.0).to(dtype)
        return x.contiguous() if self.case["layout"] == "bhld" else x.transpose(1, 2).contiguous()

    def forward(self, first):
        """The states before every chunk, the corrections U, and the state behind the last chunk."""
        B, H, dk, dv = (self.case[k] for k in ("B", "H", "dk", "dv"))
        S = torch.zeros(B, H, dk, dv, device="cuda") if first is None else first
        states, U = [], []
        for c in range(self.n):
            R = self.beta[:, :, c] * (self.V[:, :, c] - self.gamma[:, :, c] * torch.matmul(self.K[:, :, c], S))
            states.append(S)
            U.append(torch.matmul(self.T[:, :, c], R))
            S = self.Gamma[:, :, c] * S + torch.matmul((self.left[:, :, c] * self.K[:, :, c]).transpose(2, 3), U[-1])
        return torch.stack(states, 2), torch.stack(U, 2), S


def _out(x, S, U):
    return x.back(x.scale * (x.gamma * torch.matmul(x.Q, S) + torch.matmul(x.D * torch.matmul(x.Q, x.K.transpose(3, 4)), U)), _TORCH[x.case["dtype"]])


def _plain_delta(s):
    x = _Chunks(s, ("Q", "K", "V"))
    S, U, last = x.forward(s["state"])
    return _out(x, S, U), last


def _plain_train(s):
    x = _Chunks(s, ("Q", "K", "V", "dOut"))
    S, U, last = x.forward(s["state"])
    out = _out(x, S, U)
    QK = torch.matmul(x.Q, x.K.transpose(3, 4))
    do = x.scale * x.dOut
    late = torch.matmul((x.D * QK).transpose(3, 4), do)
    G = torch.zeros_like(last) if s["dstate"] is None else s["dstate"]
    after, dR = [], []
    for c in reversed(range(x.n)):   # G: the gradient of the state behind chunk c
        after.append(G)
        dR.append(torch.matmul(x.T[:, :, c].transpose(2, 3), late[:, :, c] + x.left[:, :, c] * torch.matmul(x.K[:, :, c], G)))
        G = (x.Gamma[:, :, c] * G + torch.matmul((x.gamma[:, :, c] * x.Q[:, :, c]).transpose(2, 3), do[:, :, c])
             - torch.matmul((x.gamma[:, :, c] * x.beta[:, :, c] * x.K[:, :, c]).transpose(2, 3), dR[-1]))
    after, dR = torch.stack(after[::-1], 2), torch.stack(dR[::-1], 2)
    dV = x.beta * dR
    dbeta = (dR * (x.V - x.gamma * torch.matmul(x.K, S) - torch.matmul(x.E, U))).sum(4, keepdim=True)
    r = torch.arange(x.C, device="cuda")
    N = x.D * torch.matmul(do, U.transpose(3, 4))
    M = -(x.D * torch.matmul(dV, U.transpose(3, 4))).masked_fill(r[:, None] <= r[None, :], 0.0)
    dq = x.gamma * torch.matmul(do, S.transpose(3, 4))
    dk1, dk2 = -x.gamma * torch.matmul(dV, S.transpose(3, 4)), x.left * torch.matmul(U, after.transpose(3, 4))
    dQ = dq + torch.matmul(N, x.K)
    dK = dk1 + dk2 + torch.matmul(M, x.K) + torch.matmul(M.transpose(3, 4), x.K) + torch.matmul(N.transpose(3, 4), x.Q)
    # a weight exp(G_t - G_i) belongs to the gates behind i up to t: sums that cancel, in 64 bits
    inner = (N * QK + M * x.KK).double()
    inner = inner.sum(4) - inner.sum(3)
    spent = (dk2 * x.K).double().sum(4)
    dG = (dq * x.Q + dk1 * x.K).double().sum(4) + inner - spent
    total = spent.sum(3, keepdim=True) + (x.Gamma * S * after).double().sum((3, 4))[..., None]
    dgate = dG.flip(3).cumsum(3).flip(3) + total
    f32, dtype = torch.float32, _TORCH[x.case["dtype"]]
    grads = {"dQ": x.back(dQ, dtype), "dK": x.back(dK, dtype), "dV": x.back(dV, dtype),
             "dlog_gate": x.back(dgate, f32)[..., 0], "dbeta": x.back(dbeta, f32)[..., 0]}
    if s["state"] is not None:
        grads["dstate"] = G
    return out, last, grads


def _plain_step(s):
    S = s["state"] if s["parent"] is None else s["state"][s["parent"].long()]
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    S = torch.exp(s["log_gate"])[..., None, None] * S
    u = s["beta"][..., None] * (v - (k[..., None] * S).sum(2))
    S = S + k[..., None] * u[..., None, :]
    out = (q[..., None] * S).sum(2) * q.shape[-1] ** -0.5
    s["state_out"].copy_(S)
    return out.to(s["v"].dtype), s["state_out"]


def _plain_sample(s):
    T = s["temperature"].double()[:, None]
    greedy = T <= 0
    z = s["logits"].double() / torch.where(greedy, 1.0, T)   # 64 bits: a border between two tokens can lie close to the random number
    # the stable sort leaves equal logits in the order of their tokens
    z, token = torch.sort(z, dim=1, descending=True, stable=True)
    w = torch.exp(z - z[:, :1])
    r = torch.arange(z.shape[1], device=z.device)
    k = s["top_k"].long()[:, None]
    w = torch.where((r < torch.where(greedy, 1, torch.where(k > 0, k, z.shape[1]))), w, 0.0)
    before = torch.cumsum(w, 1) - w
    p = s["top_p"].double()[:, None]
    kept = (w > 0) & ((p >= 1) | (before < p * w.sum(1, keepdim=True)) | (r == 0)) & (w >= s["min_p"].double()[:, None])
    w = torch.zeros_like(w).scatter_(1, token, torch.where(kept, w, 0.0))   # in the order of the tokens
    behind = torch.cumsum(w, 1)
    total = behind[:, -1:]
    at = (behind <= s["uniform"].double()[:, None] * total).sum(1, keepdim=True)
    return at[:, 0].to(torch.int32), torch.log(torch.gather(w, 1, at) / total)[:, 0].float()


# ---------------------------------------------------------------------------
# the definitions in 64 bits: token after token
# ---------------------------------------------------------------------------
def _exact_attention(case, s):
    B, H, L, dk, dv = (case[k] for k in ("B", "H", "L", "dk", "dv"))
    train = case["kind"] == "train"
    by_row = lambda x: (x.permute(2, 0, 1, *range(3, x.dim())) if case["layout"] == "bhld" else x.transpose(0, 1)).double().contiguous()
    q, k, v, a, beta = (by_row(s[x]) for x in ("Q", "K", "V", "log_gate", "beta"))
    a = torch.exp(a)
    length = torch.full((B,), L, device="cuda") if s["lengths"] is None else s["lengths"].long()
    scale = dk ** -0.5
    S = torch.zeros(B, H, dk, dv, dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()
    out, states, errors = torch.zeros_like(v), [], []

    def live(t):
        return (t < length)[:, None, None, None]

    for t in range(L):
        D = a[t][..., None, None] * S
        e = v[t] - torch.matmul(k[t][:, :, None], D)[:, :, 0]
        new = D + k[t][..., None] * (beta[t][..., None] * e)[:, :, None]
        if train:
            states.append(S)
            errors.append(e)
        S = torch.where(live(t), new, S)
        out[t] = torch.where(live(t)[..., 0], scale * torch.matmul(q[t][:, :, None], S)[:, :, 0], 0.0)
    back = lambda x: (x.permute(1, 2, 0, *range(3, x.dim())) if case["layout"] == "bhld" else x.transpose(0, 1)).contiguous()
    if not train:
        return back(out), S
    last, do = S, by_row(s["dOut"])
    dq, dk_, dv_, da, db = (torch.zeros_like(x) for x in (q, k, v, a, beta))
    G = torch.zeros_like(S) if s["dstate"] is None else s["dstate"].double()
    for t in reversed(range(L)):
        D, e = a[t][..., None, None] * states[t], errors[t]
        u = beta[t][..., None] * e
        new = D + k[t][..., None] * u[:, :, None]
        own_G = G + scale * q[t][..., None] * do[t][:, :, None]
        du = torch.matmul(k[t][:, :, None], own_G)[:, :, 0]
        de = beta[t][..., None] * du
        dD = own_G - k[t][..., None] * de[:, :, None]
        on = live(t)[..., 0]
        dq[t] = torch.where(on, scale * torch.matmul(new, do[t][..., None])[..., 0], 0.0)
        dk_[t] = torch.where(on, torch.matmul(own_G, u[..., None])[..., 0] - torch.matmul(D, de[..., None])[..., 0], 0.0)
        dv_[t] = torch.where(on, de, 0.0)
        db[t] = torch.where(on[..., 0], (du * e).sum(2), 0.0)
        da[t] = torch.where(on[..., 0], (dD * D).sum((2, 3)), 0.0)
        G = torch.where(live(t), a[t][..., None, None] * dD, G)
    grads = {"dQ": back(dq), "dK": back(dk_), "dV": back(dv_), "dlog_gate": back(da), "dbeta": back(db)}
    if s["state"] is not None:
        grads["dstate"] = G
    return back(out), last, grads


def _exact_sample(case, s):
    tokens, logs = [], []
    for b in range(case["B"]):
        x, T = s["logits"][b].double(), float(s["temperature"][b])
        top = float(x.max())
        if T <= 0:
            tokens.append(int(torch.nonzero(x == top)[0]))
            logs.append(0.0)
            continue
        p = torch.exp((x - top) / T)
        k, top_p, min_p = int(s["top_k"][b]), float(s["top_p"][b]), float(s["min_p"][b])
        kept = p > 0
        if 0 < k < case["V"]:
            edge = torch.topk(x, k).values[-1]
            kept &= x >= edge
            surplus = int(kept.sum()) - k   # of those that equal the k-th, the last ones
            if surplus > 0:
                kept[torch.nonzero(x == edge)[:, 0].flip(0)[:surplus]] = False
        if top_p < 1:
            mass = top_p * float(p[kept].sum())
            at = torch.nonzero(kept)[:, 0]
            # the likeliest first, equal ones by their token
            order = at[torch.sort(x[at], descending=True, stable=True).indices]
            reached = torch.cumsum(p[order], 0) >= mass
            kept[order[int(torch.nonzero(reached)[0]) + 1:]] = False
        kept &= p >= min_p
        at = torch.nonzero(kept)[:, 0]
        sums = torch.cumsum(p[at], 0)
        i = int((sums <= float(s["uniform"][b]) * sums[-1]).sum())
        tokens.append(int(at[i]))
        logs.append(float(torch.log(p[at[i]] / sums[-1])))
    return torch.tensor(tokens, dtype=torch.int32), torch.tensor(logs, dtype=torch.float64)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("delta", "train"):
        return _exact_attention(case, s)
    if case["kind"] == "sample":
        return _exact_sample(case, s)
    B = case["B"]
    rows = range(B) if s["parent"] is None else s["parent"].tolist()
    states, outs = [], []
    for b, r in enumerate(rows):
        D = torch.exp(s["log_gate"][b].double())[:, None, None] * s["state"][r].double()
        k, v = s["k"][b].double(), s["v"][b].double()
        u = s["beta"][b].double()[:, None] * (v - torch.einsum("hi,hij->hj", k, D))
        states.append(D + torch.einsum("hi,hj->hij", k, u))
        outs.append(torch.einsum("hi,hij->hj", s["q"][b].double(), states[-1]) / math.sqrt(case["dk"]))
    return torch.stack(outs), torch.stack(states)


def work(case):
    kind = case["kind"]
    size = 4 if case["dtype"] == "f32" else 2
    if kind in ("delta", "train"):
        B, H, L, dk, dv = (case[k] for k in ("B", "H", "L", "dk", "dv"))
        n, state = B * H * L, 4 * B * H * dk * dv
        # forward: a token reads the state by its key, corrects it, and reads it by its query
        moved, flops = n * (2 * (dk + dv) * size + 8) + state * (2 if case["carried"] else 1), n * 6 * dk * dv
        if kind == "train":   # the state again, its gradient (corrected, read by the key), and five readouts
            moved += n * ((4 * dk + 3 * dv) * size + 16) + (3 * state if case["carried"] else 0)
            flops += n * 18 * dk * dv
        return {"bytes": moved, "flops": flops}
    if kind == "step":
        B, H, dk, dv = (case[k] for k in ("B", "H", "dk", "dv"))
        return {"bytes": B * H * (8 * dk * dv + 2 * (dk + dv) * size + 8), "flops": B * H * 7 * dk * dv}
    B, V = case["B"], case["V"]
    return {"bytes": B * (V * size + 28), "flops": B * V * 4}
