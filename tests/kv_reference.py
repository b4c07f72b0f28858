"""Plain 64-bit forms of the paged key/value cache and of attention over a shared prefix, and the error bounds that the
kernels are held to.  Nothing here comes from the library."""
from __future__ import annotations

import math

import torch

CODE_MAX = {"e4m3": 448.0, "int8": 127.0}
CODE_TYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def quantise(x: torch.Tensor, fmt: str):
    """(codes, scales) of vectors along the last axis.  The definition's three binary32 steps are each evaluated in binary64
    and rounded once: a quotient or product of binary32 numbers rounded twice that way is rounded correctly.  A vector that
    holds an infinity or a NaN has a NaN scale and codes that say nothing."""
    x = x.float().double()
    amax = x.abs().amax(-1).clamp_min(float(torch.tensor(1e-12, dtype=torch.float32)))
    scale, inverse = (amax / CODE_MAX[fmt]).float(), (CODE_MAX[fmt] / amax).float()
    scale = torch.where(torch.isfinite(amax), scale, math.nan)
    y = torch.nan_to_num((x * inverse.double().unsqueeze(-1)).float(), nan=0.0)
    if fmt == "int8":
        return torch.round(y.double()).to(torch.int8), scale
    return y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn), scale


def same(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Equal bit for bit, any NaN being like any other."""
    ints = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[a.element_size()]
    nan = torch.isnan(a.float())
    return torch.equal(nan, torch.isnan(b.float())) and torch.equal(a.contiguous().view(ints)[~nan], b.contiguous().view(ints)[~nan])


def dequantise(codes: torch.Tensor, scale: torch.Tensor | None) -> torch.Tensor:
    x = codes.float().double()
    return x if scale is None else x * scale.double().unsqueeze(-1)


def attend(k, v, prefix_pages, prefix_len, page_table, lens, q, scale):
    """k, v: dequantised binary64 [pages, page_size, kv_heads, dim]; q [seqs, q_len, heads, dim] in its own type.  Returns
    binary64 (out, lse, weighted mean of |v|, largest sum of |q k| times |scale| over the seen keys, keys seen)."""
    seqs, q_len, heads, dim = q.shape
    page_size, kv_heads = k.shape[1], k.shape[2]
    group = heads // kv_heads
    q = q.double()
    out = torch.zeros(seqs, q_len, heads, dim, dtype=torch.float64)
    lse = torch.full((seqs, q_len, heads), -math.inf, dtype=torch.float64)
    mean_abs, score_abs, seen = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(lse)
    for b in range(seqs):
        n = int(lens[b])
        if n < 0:
            continue
        where = [(int(prefix_pages[i // page_size]), i % page_size) for i in range(prefix_len)]
        where += [(int(page_table[b][i // page_size]), i % page_size) for i in range(n)]
        pages = torch.tensor([w[0] for w in where], dtype=torch.int64)
        offsets = torch.tensor([w[1] for w in where], dtype=torch.int64)
        for i in range(q_len):
            sees = prefix_len + max(0, min(n, n - q_len + i + 1))
            if sees == 0:
                continue
            kk, vv = k[pages[:sees], offsets[:sees]], v[pages[:sees], offsets[:sees]]
            for h in range(heads):
                kh, vh = kk[:, h // group], vv[:, h // group]
                s = kh @ q[b, i, h] * scale
                lse[b, i, h] = torch.logsumexp(s, 0)
                w = torch.exp(s - lse[b, i, h])
                out[b, i, h] = w @ vh
                mean_abs[b, i, h] = w @ vh.abs()
                score_abs[b, i, h] = (kh.abs() @ q[b, i, h].abs()).max() * abs(scale)
                seen[b, i, h] = sees
    return out, lse, mean_abs, score_abs, seen


def out_tolerance(ref, mean_abs, score_abs, seen, dtype, quantised, dim):
    """Largest |out - ref| that the arithmetic allows.

    Weights are rounded to the type of the second product before it (the model's type for a plain cache, fp16 for a
    quantised one): half a step, eps / 2 relative.  A score is a binary32 sum of `dim` exact products, off by at most
    dim * 2^-24 * sum |q k|, which as an exponent is a relative error of the weight of the same size; exponentials (2^-22),
    the sums over the keys ((keys + 64) * 2^-24, numerator and denominator), the join of the parts and the division add the
    rest.  All that acts on sum w |v| / sum w.  The result is rounded to the type once: eps / 2 of its magnitude.
    fp16 weights below 2^-14 are off by up to 2^-25 of the largest, times |code| <= 448, relative to a row whose
    largest value scale is that of the largest weight: keys * 2^-25 * 448 / 127 of the largest |v| at most, bounded here
    by the largest mean."""
    product = torch.finfo(torch.float16 if quantised else dtype).eps / 2
    rest = 2.0 ** -24 * (4 * dim * score_abs + 2 * (seen + 64) + 16)
    tol = (product + rest.unsqueeze(-1)) * mean_abs + torch.finfo(dtype).eps / 2 * ref.abs() * (1 + product)
    if quantised:
        tol = tol + (seen * 2.0 ** -25 * 4).unsqueeze(-1) * mean_abs.amax(-1, keepdim=True)
    tiny = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -126  # gradual underflow of the output
    return tol + tiny


def lse_tolerance(ref, score_abs, seen, dim):
    """A score's own error, the relative error of the sum (keys * 2^-24 and the exponentials), the rounding of the result."""
    return 2.0 ** -24 * (4 * dim * score_abs + 2 * (seen + 64) + 16 + 4 * torch.nan_to_num(ref, neginf=0.0).abs())
