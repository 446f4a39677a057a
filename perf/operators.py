"""Timed cases of the readout operators: learning a readout of spike features by
the gated delta rule, and drawing decisions from scores.

**Delta rule.**  Per sequence b and value head h (an associative memory S of
dk x dv weights), sample t has a key k_t, a value v_t, a query q_t, a rate
beta_t and a log decay g_t:

    u_t = beta_t (v_t - e^{g_t} S_{t-1}^T k_t)     S_t = e^{g_t} S_{t-1} + k_t u_t^T
    out_t = scale S_t^T q_t

Keys and queries have Hk heads, and value head h reads key head h // (Hv / Hk).
Kinds: ``delta`` (a whole ordered batch in one call), ``step`` (one sample per
sequence, the memory updated in place) and ``train`` (the batch call and its
backward pass).

**Draw.**  Per row, scores below a temperature, the top_k largest, of these the
shortest run from the largest that holds top_p of the probability, of these the
ones with at least min_p times the largest probability; a given uniform number
picks one of what is left, in index order.  Equal scores are ordered by index,
masked scores are never drawn, and a row without any gives no winner.  Kind
``draw``: the winner of a layer's C x H x W neurons (or of a plain row of C
scores).
"""
import math

import torch

own = False

DEV = "cuda"
F32, F64, BF16 = torch.float32, torch.float64, torch.bfloat16
CHUNK = 64


# ------------------------------------------------------------------ the cases
def _delta(name, kind, B, L, Hk, Hv, dk, dv, bf16=False, ragged=False):
    return {"name": name, "kind": kind, "B": B, "L": L, "Hk": Hk, "Hv": Hv, "dk": dk, "dv": dv, "bf16": bf16,
            "ragged": ragged}


def _pick(name, B, C, H, W, bf16, temperature, top_k, top_p, min_p, masked):
    return {"name": name, "kind": "draw", "B": B, "C": C, "H": H, "W": W, "bf16": bf16, "temperature": temperature,
            "top_k": top_k, "top_p": top_p, "min_p": min_p, "masked": masked}


def listed():
    return [
        # one group of the online trainer: 16 images, 200 maps' features onto 10 classes
        _delta("delta_16x200x10", "delta", 1, 16, 1, 1, 200, 10),
        # the benchmark's batch of 1000 images in one ordered replay, 8 readouts of 250 features
        _delta("delta_b1000_250x10", "delta", 1, 1000, 8, 8, 250, 10),
        # long sequences, many memories, two to a key head
        _delta("delta_4x4096_bf16", "delta", 4, 4096, 16, 32, 128, 128, True),
        # a padded batch of sequences from none to 1531 samples, odd sizes
        _delta("delta_ragged_bf16", "delta", 8, 1531, 4, 8, 96, 72, True, True),
        # one image after another: a single small readout, latency alone
        _delta("step_1x250x10", "step", 1, 1, 1, 8, 250, 10),
        # one sample of each of 256 sequences: the memories are read and written once
        _delta("step_256_bf16", "step", 256, 1, 16, 32, 128, 128, True),
        # gradients of a small readout over a batch
        _delta("train_250x200x10", "train", 1, 250, 2, 4, 200, 10),
        # gradients through long sequences with shared key heads
        _delta("train_2x2048_bf16", "train", 2, 2048, 16, 32, 128, 128, True),
        # gradients of a padded batch, odd sizes
        _delta("train_ragged_bf16", "train", 5, 777, 3, 6, 65, 50, True, True),
        # the classifying layer of 1000 images: 200 maps of 4x4, silent neurons masked
        _pick("draw_b1000_200x4x4", 1000, 200, 4, 4, False, 2.0, 0, 0.9375, 0.0, True),
        # one row of many scores
        _pick("draw_1x131072_bf16", 1, 131072, 1, 1, True, 0.75, 50, 0.9375, 0.0, False),
        # a batch of long rows of an odd length, no top_k
        _pick("draw_256x200003", 256, 200003, 1, 1, False, 1.0, 0, 0.875, 0.03125, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["delta", "delta", "step", "train", "draw", "draw"])
    if kind == "draw":
        B = _log(rng, 1, 1000)
        if rng.random() < 0.4:
            H = rng.randint(1, 14)
            W = rng.randint(1, 14)
            C = _log(rng, 10, 1000)
        else:
            H = W = 1
            C = _log(rng, 1000, max(2000, min(250000, 50000000 // B)))
        c = _pick("", B, C, H, W, rng.random() < 0.5, rng.choice([0.5, 0.75, 1.0, 2.0]), rng.choice([0, 0, 1, 20, 50, 400]),
                  rng.choice([1.0, 0.5, 0.875, 0.9375]), rng.choice([0.0, 0.0, 0.03125, 0.125]), rng.random() < 0.5)
    else:
        Hk = rng.choice([1, 2, 3, 4, 8, 16])
        Hv = Hk * rng.choice([1, 1, 2, 3])
        bf16 = rng.random() < 0.6
        dk = rng.randint(16, 256)
        dv = rng.choice([10, rng.randint(5, 128), rng.randint(5, 256)])
        if kind == "step":
            B, L = _log(rng, 1, 256), 1
        else:
            B = _log(rng, 1, 8)
            most = (4 << 30 if kind == "train" else 16 << 30) // (B * Hv * dk * dv * (1 if bf16 else 2))
            L = _log(rng, 1, max(2, min(2048 if kind == "train" else 4096, most)))
        c = _delta("", kind, B, L, Hk, Hv, dk, dv, bf16, kind != "step" and rng.random() < 0.4)
    del c["name"]
    return c


def _lengths(c):
    """Sequence lengths of a padded batch: none, one, and on to L."""
    B, L = c["B"], c["L"]
    if not c["ragged"]:
        return [L] * B
    n = [min(L, 1 + (L - 1) * i // max(1, B - 1)) for i in range(B)]
    if B > 2:
        n[1] = 0
    n[-1] = L
    return n


# ------------------------------------------------------------------ inputs
def prepare(c, seed):
    r = torch.Generator(device=DEV)
    r.manual_seed(seed)

    def randn(*s):
        return torch.randn(s, generator=r, device=DEV, dtype=F32)

    def rand(*s):
        return torch.rand(s, generator=r, device=DEV, dtype=F32)

    if c["kind"] == "draw":
        shape = (c["B"], c["C"], c["H"], c["W"])
        # a layer's potentials lie above 0, a readout's scores around 0
        x = randn(*shape).abs() * 6 if c["masked"] else randn(*shape) * 2.5
        s = {"c": c, "scores": x.to(BF16) if c["bf16"] else x, "u": rand(c["B"]), "t_first": None}
        if c["masked"]:  # silent neurons, and now and then a silent image
            tf = torch.where(rand(*shape) < 0.4, 14, 15)
            tf[rand(c["B"]) < 0.03] = 15
            s["t_first"] = tf.to(torch.uint8)
        return s
    B, L, Hk, Hv, dk, dv = (c[n] for n in ("B", "L", "Hk", "Hv", "dk", "dv"))
    T = BF16 if c["bf16"] else F32
    if c["bf16"]:  # dense keys, queries and values
        k, q, v = randn(B, L, Hk, dk), randn(B, L, Hk, dk), randn(B, L, Hv, dv)
    else:  # spike features (not negative), the classes as values
        k, q = randn(B, L, Hk, dk).clamp_(min=0), randn(B, L, Hk, dk).clamp_(min=0)
        v = torch.zeros(B, L, Hv, dv, device=DEV)
        v.scatter_(3, torch.randint(0, dv, (B, L, Hv, 1), generator=r, device=DEV), 1.0)
    k, q = (x / x.norm(dim=-1, keepdim=True).clamp(min=1e-6) for x in (k, q))
    s = {"c": c, "q": q.to(T), "k": k.to(T), "v": v.to(T), "scale": 1.0,
         "beta": torch.sigmoid(randn(B, L, Hv)), "g": -torch.exp(rand(B, L, Hv) * 7.5 - 8),
         "state": randn(B, Hv, dk, dv) * 0.1, "lengths": None}
    if c["ragged"]:
        s["lengths"] = torch.tensor(_lengths(c), dtype=torch.int32, device=DEV)
    if c["kind"] == "step":
        s.update({n: s[n][:, 0].contiguous() for n in ("q", "k", "v", "beta", "g")})
    if c["kind"] == "train":
        s["d_out"] = randn(B, L, Hv, dv).to(T)
        s["d_state"] = randn(B, Hv, dk, dv) * 0.1
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    return {"delta": _run_delta, "step": _run_step, "train": _run_train, "draw": _run_draw}[s["c"]["kind"]](s)


def _run_delta(s):
    if own:
        from paper_1903_02440_amd import spk_delta_rule
        return spk_delta_rule(s["q"], s["k"], s["v"], s["g"], s["beta"], scale=s["scale"], initial_state=s["state"],
                              lengths=s["lengths"])
    out, state = _chunks(s["q"].float(), s["k"].float(), s["v"].float(), s["g"], s["beta"], s["scale"], s["state"],
                         s["lengths"])
    return out.to(s["q"].dtype), state


def _run_step(s):
    if own:
        from paper_1903_02440_amd import spk_delta_rule_step
        return spk_delta_rule_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["state"], scale=s["scale"]), s["state"]
    S, n = s["state"], s["c"]["Hv"] // s["c"]["Hk"]
    k = s["k"].float().repeat_interleave(n, 1).unsqueeze(-1)
    q = s["q"].float().repeat_interleave(n, 1).unsqueeze(-1)
    S.mul_(torch.exp(s["g"])[..., None, None])
    u = s["beta"][..., None] * (s["v"].float() - (S * k).sum(2))
    S.add_(k * u.unsqueeze(2))
    return ((S * q).sum(2) * s["scale"]).to(s["q"].dtype), S


def _run_train(s):
    if own:
        from paper_1903_02440_amd import spk_delta_rule, spk_delta_rule_backward
        a = (s["q"], s["k"], s["v"], s["g"], s["beta"])
        out, state = spk_delta_rule(*a, scale=s["scale"], initial_state=s["state"], lengths=s["lengths"])
        return (out, state) + tuple(spk_delta_rule_backward(*a, s["d_out"], d_final_state=s["d_state"],
                                                            scale=s["scale"], initial_state=s["state"],
                                                            lengths=s["lengths"]))
    x = [s[n].detach().float().requires_grad_() for n in ("q", "k", "v", "g", "beta", "state")]
    out, state = _chunks(*x[:5], s["scale"], x[5], s["lengths"])
    grads = torch.autograd.grad([out, state], x, [s["d_out"].float(), s["d_state"]])
    T = s["q"].dtype
    return (out.detach().to(T), state.detach()) + tuple(d.to(T) if i < 3 else d for i, d in enumerate(grads))


def _run_draw(s):
    c = s["c"]
    if own:
        from paper_1903_02440_amd import spk_sample_winners
        return spk_sample_winners(s["scores"], s["u"], temperature=c["temperature"], top_k=c["top_k"],
                                  top_p=c["top_p"], min_p=c["min_p"], t_first=s["t_first"], T=15)
    B, C, H, W = s["scores"].shape
    x = s["scores"].reshape(B, -1).double()
    tf = s["t_first"]
    if tf is not None:
        tf = tf.reshape(B, -1)
        x = torch.where(tf < 15, x, -math.inf)
    v, order = x.sort(dim=1, descending=True, stable=True)
    some = v[:, :1] > -math.inf
    w = torch.where(v == v[:, :1], 1.0, torch.exp((v - v[:, :1]) / c["temperature"]))
    keep = (v > -math.inf) & some
    if c["top_k"] > 0:
        keep[:, c["top_k"]:] = False
    w = torch.where(keep, w, 0.0)
    cum = w.cumsum(1)
    if c["top_p"] < 1:
        keep &= cum - w < c["top_p"] * cum[:, -1:]
    keep &= w >= c["min_p"]
    w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))
    cum = w.cumsum(1)
    at = (cum <= s["u"].double()[:, None] * cum[:, -1:]).sum(1, keepdim=True).clamp(max=C * H * W - 1)
    t = tf.gather(1, at).long() if tf is not None else torch.zeros_like(at)
    win = torch.cat([at // (H * W), t, at // W % H, at % W], 1)
    return torch.where(some, win, -1).to(torch.int32).reshape(B, 1, 4), some.reshape(-1).to(torch.int32)


def _chunks(q, k, v, g, beta, scale, S, lengths):
    """The delta rule over chunks of 64 samples.  With gamma the decays' running
    sum in a chunk, D_ij = e^{gamma_i - gamma_j} for j <= i and S the memory that
    enters it, U solves (I + A) U = beta (V - e^gamma K S) with A_ij =
    beta_i D_ij k_i.k_j for j < i; then out = e^gamma Q S + (D Q K^T) U, and
    the memory leaves as e^{gamma_C} S + (e^{gamma_C - gamma} K)^T U."""
    B, L, Hv, dv = v.shape
    n = Hv // q.shape[2]
    if lengths is not None:
        live = (torch.arange(L, device=DEV) < lengths[:, None])[:, :, None]
        q, k, v = (torch.where(live[..., None], x, 0.0) for x in (q, k, v))
        g, beta = torch.where(live, g, 0.0), torch.where(live, beta, 0.0)
    N = -(-L // CHUNK)

    def cut(x):  # [B, L, H, ...] -> [B, Hv, N, CHUNK, ...]
        x = torch.nn.functional.pad(x, (0, 0) * (x.dim() - 2) + (0, N * CHUNK - L))
        x = x.repeat_interleave(Hv // x.shape[2], 2)
        return x.transpose(1, 2).reshape(B, Hv, N, CHUNK, *x.shape[3:])

    q, k, v, g, beta = (cut(x) for x in (q, k, v, g, beta))
    gamma = g.double().cumsum(-1)
    lower = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=DEV).tril()
    D = torch.exp((gamma[..., :, None] - gamma[..., None, :]).masked_fill(~lower, -math.inf)).float()
    E = torch.exp(gamma).float()[..., None]
    last = torch.exp(gamma[..., -1:] - gamma).float()[..., None]
    b = beta[..., None]
    kt = k.transpose(-1, -2).contiguous()
    A = (b * D * (k @ kt)).tril(-1) + torch.eye(CHUNK, device=DEV)
    P, Q, K, Kl = D * (q @ kt), E * q, E * k, (last * k).transpose(-1, -2).contiguous()
    out = []
    for i in range(N):
        U = torch.linalg.solve_triangular(A[:, :, i], b[:, :, i] * (v[:, :, i] - K[:, :, i] @ S), upper=False,
                                          unitriangular=True)
        out.append(Q[:, :, i] @ S + P[:, :, i] @ U)
        S = E[:, :, i, -1:] * S + Kl[:, :, i] @ U
    out = torch.stack(out, 2).reshape(B, Hv, N * CHUNK, dv)[:, :, :L].transpose(1, 2)
    return scale * out, S


# ------------------------------------------------------------------ work
def work(c):
    if c["kind"] == "draw":
        n = c["B"] * c["C"] * c["H"] * c["W"]
        # each score read once and weighed once (a difference, an exponential, a sum)
        return {"bytes": n * ((2 if c["bf16"] else 4) + (1 if c["masked"] else 0)) + 24 * c["B"], "flops": 4 * n}
    e = 2 if c["bf16"] else 4
    tokens, cell = sum(_lengths(c)), c["dk"] * c["dv"]
    rows = tokens * (2 * c["Hk"] * c["dk"] + 2 * c["Hv"] * c["dv"]) * e + tokens * c["Hv"] * 8
    states = 2 * c["B"] * c["Hv"] * cell * 4
    # S^T k, k u^T and S^T q: 2 dk dv each; the backward pass has S^T k and k u^T again and seven more
    flops = 6 * tokens * c["Hv"] * cell
    if c["kind"] == "train":
        rows, states, flops = 2 * rows + tokens * c["Hv"] * c["dv"] * e, 2 * states, flops + 18 * tokens * c["Hv"] * cell
    return {"bytes": rows + states, "flops": flops}


# ------------------------------------------------------------------ 64 bits
def _recur(q, k, v, g, beta, scale, S, live, keep=0):
    """One sample after another in 64 bits, as the definition reads; every `keep` samples the memory is kept too."""
    outs, kept = [], []
    n = v.shape[2] // q.shape[2]
    for t in range(q.shape[1]):
        if keep and t % keep == 0:
            kept.append(S)
        kt, qt = (x[:, t].repeat_interleave(n, 1) for x in (k, q))
        on = live[:, t, None]
        S1 = S * torch.exp(torch.where(on, g[:, t], 0.0))[..., None, None]
        err = v[:, t] - torch.einsum("bhk,bhkv->bhv", kt, S1)
        u = torch.where(on, beta[:, t], 0.0)[..., None] * err
        S = S1 + kt[..., None] * u[..., None, :]
        outs.append(scale * torch.where(on[..., None], torch.einsum("bhk,bhkv->bhv", qt, S), 0.0))
    return torch.stack(outs, 1), S, kept


def exact(c, seed):
    if c["kind"] == "draw":
        return None  # whole numbers
    s = prepare(c, seed)
    x = [s[n].double() for n in ("q", "k", "v", "g", "beta")]
    S = s["state"].double()
    if c["kind"] == "step":
        x = [a[:, None] for a in x]
    live = torch.arange(x[0].shape[1], device=DEV)[None] < torch.tensor(_lengths(c), device=DEV)[:, None]
    with torch.no_grad():
        out, last, kept = _recur(*x, s["scale"], S, live, keep=32)
    if c["kind"] == "step":
        return out[:, 0], last
    if c["kind"] == "delta":
        return out, last
    # backwards by runs of 32 samples from the memories kept before each
    grads, d, do = [], s["d_state"].double(), s["d_out"].double()
    for i in reversed(range(len(kept))):
        at = slice(32 * i, 32 * i + 32)
        leaf = [a[:, at].detach().requires_grad_() for a in x] + [kept[i].detach().requires_grad_()]
        o, e, _ = _recur(*leaf[:5], s["scale"], leaf[5], live[:, at])
        *part, d = torch.autograd.grad([o, e], leaf, [do[:, at], d])
        grads.append(part)
    return (out, last) + tuple(torch.cat(p[::-1], 1) for p in zip(*grads)) + (d,)
