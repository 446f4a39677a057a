"""Plain 64-bit forms of the readout operators, as their definitions read, on the
CPU (the tests' reference; nothing of the package is used)."""
import math

import numpy as np
import torch


def delta_rule(q, k, v, g, beta, scale, state, lengths=None):
    """One sample after another; tensors of any float type -> (out, final state) in float64, differentiable."""
    B, L, Hv, dv = v.shape
    n = Hv // q.shape[2]
    dk = q.shape[3]
    q, k, v, g, beta = (x.double().cpu() if not x.requires_grad else x for x in (q, k, v, g, beta))
    S = torch.zeros(B, Hv, dk, dv, dtype=torch.float64) if state is None else state
    S = S if S.requires_grad else S.double().cpu()
    lens = [L] * B if lengths is None else [max(0, min(L, int(m))) for m in lengths]
    q, k = q.repeat_interleave(n, 2), k.repeat_interleave(n, 2)
    outs, finals = [], []
    for b in range(B):
        s, rows = S[b], []
        for t in range(lens[b]):
            s = s * torch.exp(g[b, t])[:, None, None]
            u = beta[b, t][:, None] * (v[b, t] - torch.einsum("hk,hkv->hv", k[b, t], s))
            s = s + k[b, t][:, :, None] * u[:, None, :]
            rows.append(scale * torch.einsum("hk,hkv->hv", q[b, t], s))
        rows += [torch.zeros(Hv, dv, dtype=torch.float64)] * (L - lens[b])
        outs.append(torch.stack(rows) if rows else torch.zeros(0, Hv, dv, dtype=torch.float64))
        finals.append(s)
    return torch.stack(outs), torch.stack(finals)


def sample_winners(scores, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, t_first=None, T=1):
    """Step by step as the definition reads, with the weights as 64-bit floats summed exactly."""
    scores = np.asarray(scores, np.float64)
    B, C, H, W = scores.shape
    win, n_win = np.full((B, 1, 4), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        x = scores[b].reshape(-1)
        ok = ~np.isnan(x) & (x > -math.inf)
        if t_first is not None:
            ok &= np.asarray(t_first[b]).reshape(-1) < T
        idx = np.nonzero(ok)[0]
        if not len(idx):
            continue
        order = idx[np.argsort(-x[idx], kind="stable")]
        if temperature == 0:
            order = order[:1]
        elif top_k:
            order = order[:top_k]
        top = x[order[0]]
        w = [1.0 if x[i] == top else math.exp((x[i] - top) / temperature) for i in order]
        if top_p < 1 and temperature > 0:
            total, run, m = math.fsum(w), 0.0, 0
            for m in range(1, len(w) + 1):
                run = math.fsum([run, w[m - 1]])
                if run >= top_p * total:
                    break
            order, w = order[:m], w[:m]
        kept = sorted((i, wi) for i, wi in zip(order, w) if wi >= min_p)
        total, run = math.fsum(wi for _, wi in kept), 0.0
        ub = float(u[b])
        ub = 0.0 if math.isnan(ub) else min(max(ub, 0.0), 1.0)
        at = kept[-1][0]
        for i, wi in kept:
            run = math.fsum([run, wi])
            if run > ub * total:
                at = i
                break
        win[b, 0] = (at // (H * W), 0 if t_first is None else np.asarray(t_first[b]).reshape(-1)[at],
                     at // W % H, at % W)
        n_win[b] = 1
    return win, n_win
