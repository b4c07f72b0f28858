"""The plain 64-bit form of attention over packed prompts.  Nothing here comes from the library."""
from __future__ import annotations

import math

import torch


def attend(q, k, v, q_starts, k_starts, causal, scale):
    """q [q_tokens, heads, dim], k, v [k_tokens, kv_heads, dim] in their own types.  Returns binary64 (out, lse, weighted mean of |v|,
    largest sum of |q k| times |scale| over the seen keys, keys seen, rows of some sequence), as kv_reference.out_tolerance wants them."""
    heads, dim = q.shape[1:]
    kv_heads = k.shape[1]
    group = heads // kv_heads
    q, k, v = q.double(), k.double(), v.double()
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    mean_abs, score_abs, seen = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(lse)
    live = torch.zeros(q.shape[0], dtype=torch.bool)
    for b in range(len(q_starts) - 1):
        (q0, q1), (k0, k1) = (q_starts[b], q_starts[b + 1]), (k_starts[b], k_starts[b + 1])
        n_q, n_k = q1 - q0, k1 - k0
        if n_q <= 0:
            continue
        live[q0:q1] = True
        if n_k <= 0:
            continue
        i, j = torch.arange(n_q)[:, None], torch.arange(n_k)[None]
        hidden = (j > n_k - n_q + i) if causal else torch.zeros(n_q, n_k, dtype=torch.bool)
        some = ~hidden.all(1)
        for h in range(heads):
            kh, vh, qh = k[k0:k1, h // group], v[k0:k1, h // group], q[q0:q1, h]
            s = (qh @ kh.T * scale).masked_fill(hidden, -math.inf)
            total = torch.logsumexp(s, 1)
            w = torch.where(some[:, None], torch.exp(s - torch.where(some, total, 0.0)[:, None]), 0.0)
            rows = slice(q0, q1)
            lse[rows, h] = torch.where(some, total, -math.inf)
            w0 = w.masked_fill(hidden, 0.0)
            finite = torch.isfinite(vh).all()
            out[rows, h] = w0 @ vh if finite else _careful(w0, hidden, vh)
            mean_abs[rows, h] = w0 @ torch.nan_to_num(vh, nan=0.0, posinf=0.0, neginf=0.0).abs()
            score_abs[rows, h] = (qh.abs() @ kh.abs().T * abs(scale)).masked_fill(hidden, 0.0).amax(1)
            seen[rows, h] = (~hidden).sum(1).double()
    return out, lse, mean_abs, score_abs, seen, live


def _careful(w, hidden, v):
    """The product with values that are not all finite: those of hidden keys count nothing."""
    out = torch.zeros(w.shape[0], v.shape[1], dtype=torch.float64)
    for i in range(w.shape[0]):
        out[i] = w[i, ~hidden[i]] @ v[~hidden[i]]
    return out
