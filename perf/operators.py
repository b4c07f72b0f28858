"""Cases of the serving-side attention operators: a paged key/value cache that is quantised as it is written, the same
cache read back, and attention for a batch of sequences that share a long prefix.

``own`` is False: ``run`` computes the plain form (elementary torch operations in 32 bits).  Where it is True, ``run``
makes the calls of the package's binding that a serving program makes.

Definitions.  A cache is a set of pages of ``page`` tokens; the entry of a token and head is a vector of ``dim`` values.
Plain caches hold the model's type.  Quantised caches hold codes and one binary32 scale per token and head, apart for
keys and values: amax = max(max |x|, 1e-12), scale = amax / M, code = round_to_nearest_even(x * (M / amax)), each step a
binary32 operation, M = 448 for e4m3 codes and 127 for int8 codes; the value read back is code * scale.  A slot number is
page * page_size + offset; a negative one marks a padded token, which is skipped.

Attention.  Every sequence attends to the keys of the prefix, then to those of its own suffix, whose last ``q_len`` keys
are the query tokens' own (query i of sequence b sees suffix keys j <= len_b - q_len + i).  Query head h reads
key/value head h // (heads / kv_heads).  The outputs are the attention result and the natural logarithm of the softmax
denominator (-inf and a zero row where no key is seen).  A negative suffix length marks a padded sequence, whose rows
stay as they were.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
CODE_MAX = {"e4m3": 448.0, "int8": 127.0}
CODE_TYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def _write(name, tokens, heads, dim, page, dtype, fmt, readback=False, padded=0):
    return {"name": name, "op": "write", "tokens": tokens, "kv_heads": heads, "dim": dim, "page": page, "dtype": dtype,
            "fmt": fmt, "readback": readback, "padded": padded}


def _read(name, tokens, heads, dim, page, dtype, fmt):
    return {"name": name, "op": "read", "tokens": tokens, "kv_heads": heads, "dim": dim, "page": page, "dtype": dtype, "fmt": fmt}


def _attend(name, seqs, q_len, heads, kv_heads, dim, prefix, suffix, page, dtype, fmt, padded=0):
    return {"name": name, "op": "attend", "seqs": seqs, "q_len": q_len, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "prefix": prefix, "suffix": suffix, "page": page, "dtype": dtype, "fmt": fmt, "padded": padded}


def listed():
    return [
        # the cache write of one decoding step of a batch of 64: latency counts
        _write("write_64x8x128_bf16_e4m3", 64, 8, 128, 16, "bf16", "e4m3"),
        # the write of a prefill of 16384 tokens
        _write("write_16384x8x128_bf16_e4m3", 16384, 8, 128, 64, "bf16", "e4m3"),
        # a padded batch with an odd number of heads and a head size that wide vectors do not divide; written, then read back
        _write("write_1000x5x100_fp16_int8_back", 1000, 5, 100, 16, "fp16", "int8", True, 24),
        # one sequence's context fetched out of the cache for a short chunk of prefill
        _read("read_777x8x64_fp16_int8", 777, 8, 64, 16, "fp16", "int8"),
        # a long context fetched out of the cache
        _read("read_16384x8x128_bf16_e4m3", 16384, 8, 128, 64, "bf16", "e4m3"),
        # two conversations on a short prompt: latency counts
        _attend("attend_2x1_32of8x128_p512", 2, 1, 32, 8, 128, 512, 64, 16, "bf16", "plain"),
        # verification of five drafted tokens, one head per key/value head, padded batch, lengths off the page size
        _attend("attend_17x5_8of8x64_p4097_fp16", 17, 5, 8, 8, 64, 4097, 333, 16, "fp16", "plain", 1),
        # a batch of 64 on a system prompt of 8192 tokens, e4m3 cache
        _attend("attend_64x1_32of8x128_p8192_e4m3", 64, 1, 32, 8, 128, 8192, 1024, 64, "bf16", "e4m3"),
        # five query heads per key/value head, int8 cache, a prefix that ends inside a page
        _attend("attend_48x1_40of8x128_p16001_int8", 48, 1, 40, 8, 128, 16001, 700, 32, "bf16", "int8"),
        # heads of 256
        _attend("attend_32x1_32of4x256_p2500", 32, 1, 32, 4, 256, 2500, 512, 64, "bf16", "plain"),
        # a large batch on a document of 32768 tokens
        _attend("attend_256x1_32of8x128_p32768", 256, 1, 32, 8, 128, 32768, 2048, 64, "bf16", "plain"),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["write", "read", "attend", "attend"])
    if op != "attend":
        heads, dim = rng.choice([1, 2, 4, 5, 8, 16, 32]), rng.choice([33, 64, 80, 100, 128, 256])
        dtype, page = rng.choice(["bf16", "bf16", "fp16", "fp32"]), rng.choice([1, 8, 16, 32, 64, 128])
        most = 16384 * 8 * 128 // (2 if dtype == "fp32" else 1)
        tokens = _log_uniform(rng, 1, min(16384, most // (heads * dim)))
        fmt = rng.choice(["e4m3", "e4m3", "int8", "plain"])
        case = _read("", tokens, heads, dim, page, dtype, fmt)
        if op == "write":
            case = _write("", tokens, heads, dim, page, dtype, fmt, fmt == "int8" or rng.random() < 0.3, rng.choice([0, tokens // 9]))
    else:
        kv_heads, group, dim = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([64, 64, 80, 96, 128, 128, 128, 256])
        seqs, prefix, suffix = _log_uniform(rng, 1, 256), _log_uniform(rng, 1, 32768), _log_uniform(rng, 1, 2048)
        q_len = rng.choice([1, 1, 1, 2, 5, 8])
        group = min(group, max(1, 32 // kv_heads))
        while seqs * q_len * kv_heads * group * prefix * dim > 256 * 32 * 32768 * 128 or seqs * suffix * kv_heads * dim > 256 * 2048 * 8 * 128 // 2:
            seqs = max(1, seqs // 2)
        case = _attend("", seqs, q_len, kv_heads * group, kv_heads, dim, prefix, suffix, rng.choice([1, 8, 16, 32, 64, 128]),
                       rng.choice(["bf16", "bf16", "fp16"]), rng.choice(["plain", "plain", "e4m3", "int8"]), rng.choice([0, 0, seqs // 5]))
    del case["name"]
    return case


# ---- inputs -------------------------------------------------------------------------------------------------------

def _suffix_lengths(case):
    """Suffix lengths of the batch, before they are shuffled: spread over 0 .. suffix, the padded sequences last."""
    live = case["seqs"] - case["padded"]
    lens = [round(case["suffix"] * (i + 1) / live) for i in range(live)]
    if live > 2:
        lens[0] = 0  # a sequence that has only the prefix
    return lens + [-1] * case["padded"]


def _codes(x, fmt):
    """(codes, scales) of the vectors along the last axis of binary32 x: the definition at the top of this file."""
    amax = x.abs().amax(-1).clamp_min(1e-12)
    scaled = x * (CODE_MAX[fmt] / amax).unsqueeze(-1)
    codes = scaled.to(torch.float8_e4m3fn) if fmt == "e4m3" else scaled.round().to(torch.int8)
    return codes, amax / CODE_MAX[fmt]


def _fill(shape, dtype, gen):
    """Keys and values as projections make them: channels of different strengths, a few of them strong."""
    channel = torch.exp(0.4 * torch.randn(shape[-2:], generator=gen, device="cuda"))
    return (torch.randn(shape, generator=gen, device="cuda") * channel).to(dtype)


def _new_cache(case, n_pages, gen, filled):
    shape = (n_pages, case["page"], case["kv_heads"], case["dim"])
    dtype, fmt = DTYPES[case["dtype"]], case["fmt"]
    cache = {}
    for side in ("k", "v"):
        if fmt == "plain":
            cache[side] = _fill(shape, dtype, gen) if filled else torch.zeros(shape, dtype=dtype, device="cuda")
        elif filled:
            cache[side], cache[side + "_scale"] = _codes(_fill(shape, dtype, gen).float(), fmt)
        else:
            cache[side] = torch.zeros(shape, dtype=torch.uint8, device="cuda").view(CODE_TYPE[fmt])
            cache[side + "_scale"] = torch.zeros(shape[:3], dtype=torch.float32, device="cuda")
    return cache


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    page, dtype = case["page"], DTYPES[case["dtype"]]
    state = {"case": dict(case)}
    if case["op"] in ("write", "read"):
        tokens, heads, dim = case["tokens"], case["kv_heads"], case["dim"]
        n_pages = -(-tokens // page) + 3
        # the pages of a few sequences, in the order in which an allocator handed them out
        order = torch.randperm(n_pages, generator=gen, device="cuda")
        at = torch.arange(tokens, device="cuda")
        slots = order[at // page] * page + at % page
        state["cache"] = _new_cache(case, n_pages, gen, case["op"] == "read")
        if case["op"] == "write":
            padded = case["padded"]
            state["live"] = tokens - padded
            if padded:
                slots[tokens - padded:] = -1
            # key and value as they leave the projection: slices of one [tokens, 2 * heads * dim] tensor
            both = _fill((tokens, 2 * heads, dim), dtype, gen)
            state["key"], state["value"] = both[:, :heads], both[:, heads:]
        state["slots"] = slots
        if case["op"] == "read" or case["readback"]:
            state["key_out"] = torch.zeros(tokens, heads, dim, dtype=dtype, device="cuda")
            state["value_out"] = torch.zeros(tokens, heads, dim, dtype=dtype, device="cuda")
    else:
        seqs, prefix, most = case["seqs"], case["prefix"], case["suffix"]
        lens = torch.tensor(_suffix_lengths(case), device="cuda", dtype=torch.int32)
        live = seqs - case["padded"]
        lens[:live] = lens[:live][torch.randperm(live, generator=gen, device="cuda")]
        prefix_n, width = -(-prefix // page), -(-most // page)
        per_seq = (lens.clamp_min(0) + page - 1) // page
        n_pages = prefix_n + int(per_seq.sum()) + 2
        order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        begin = prefix_n + torch.cumsum(per_seq, 0) - per_seq
        column = torch.arange(width, device="cuda")
        table = torch.where(column < per_seq.unsqueeze(1), order[(begin.unsqueeze(1) + column).clamp_max(n_pages - 1).long()], 0)
        state["prefix_pages"], state["page_table"], state["lens"] = order[:prefix_n].contiguous(), table.to(torch.int32), lens
        state["cache"] = _new_cache(case, n_pages, gen, True)
        rows = seqs * case["q_len"]
        state["q"] = torch.randn(rows, case["heads"], case["dim"], generator=gen, device="cuda").to(dtype).view(seqs, case["q_len"], case["heads"], case["dim"])
        state["out"] = torch.zeros_like(state["q"])
        state["lse"] = torch.zeros(seqs, case["q_len"], case["heads"], dtype=torch.float32, device="cuda")
        state["scale"] = 1.0 / math.sqrt(case["dim"])
    if own:
        from paper_2601_12698_b200 import binding
        c = state["cache"]
        state["binding"] = binding
        state["handle"] = binding.KvCache(c["k"], c["v"], c.get("k_scale"), c.get("v_scale"))
        if case["op"] == "attend":
            state["batch"] = binding.PrefixBatch(state["prefix_pages"], case["prefix"], state["page_table"], state["lens"], case["suffix"], case["q_len"])
            state["workspace"] = binding.shared_prefix_attention_workspace(state["handle"], state["batch"], case["heads"])
    return state


# ---- the passes -----------------------------------------------------------------------------------------------------

def _read_plain(cache, slots, dtype):
    """Entries of the cache at `slots` as [..., kv_heads, dim], keys and values."""
    got = []
    for side in ("k", "v"):
        entries = cache[side].flatten(0, 1)
        if entries.dtype == torch.float8_e4m3fn:
            x = entries.view(torch.uint8)[slots].view(torch.float8_e4m3fn).float()
        else:
            x = entries[slots].float()
        if side + "_scale" in cache:
            x = x * cache[side + "_scale"].flatten(0, 1)[slots].unsqueeze(-1)
        got.append(x.to(dtype))
    return got


def _write_plain(state):
    cache, live, fmt = state["cache"], state["live"], state["case"]["fmt"]
    slots = state["slots"][:live]
    for side, x in (("k", state["key"][:live]), ("v", state["value"][:live])):
        if fmt == "plain":
            cache[side].flatten(0, 1)[slots] = x
        else:
            codes, scales = _codes(x.float(), fmt)
            cache[side].view(torch.uint8).flatten(0, 1)[slots] = codes.view(torch.uint8)
            cache[side + "_scale"].flatten(0, 1)[slots] = scales


def _attend_plain(state):
    case, q, lens = state["case"], state["q"].float(), state["lens"].long()
    seqs, q_len, heads, dim = q.shape
    kv_heads, page, most = case["kv_heads"], case["page"], case["suffix"]
    group = heads // kv_heads
    at = torch.arange(case["prefix"], device="cuda")
    k_pre, v_pre = _read_plain(state["cache"], state["prefix_pages"].long()[at // page] * page + at % page, torch.float32)
    at = torch.arange(most, device="cuda")
    k_suf, v_suf = _read_plain(state["cache"], state["page_table"].long()[:, at // page] * page + at % page, torch.float32)
    # rows of one key/value head: its query heads of every query token
    rows = q.view(seqs, q_len, kv_heads, group, dim).permute(2, 0, 1, 3, 4) * state["scale"]            # [K, B, Q, G, d]
    s_pre = torch.matmul(rows.reshape(kv_heads, -1, dim), k_pre.permute(1, 2, 0))                       # [K, B*Q*G, prefix]
    s_suf = torch.matmul(rows.reshape(kv_heads, seqs, q_len * group, dim), k_suf.permute(2, 0, 3, 1))   # [K, B, Q*G, suffix]
    last = lens.unsqueeze(1) - q_len + torch.arange(q_len, device="cuda")                               # [B, Q]
    seen = at <= last.unsqueeze(-1)                                                                     # [B, Q, suffix]
    s_suf = s_suf.view(kv_heads, seqs, q_len, group, most).masked_fill(~seen.unsqueeze(2), float("-inf"))
    s_pre = s_pre.view(kv_heads, seqs, q_len, group, -1)
    top = torch.maximum(s_pre.amax(-1), s_suf.amax(-1))
    base = torch.where(torch.isinf(top), torch.zeros_like(top), top).unsqueeze(-1)
    e_pre, e_suf = torch.exp(s_pre - base), torch.exp(s_suf - base)
    total = e_pre.sum(-1) + e_suf.sum(-1)
    o = torch.matmul(e_pre.view(kv_heads, -1, s_pre.shape[-1]), v_pre.permute(1, 0, 2)).view(kv_heads, seqs, q_len, group, dim)
    v_suf = v_suf.masked_fill(~(at < lens.unsqueeze(1))[..., None, None], 0.0)
    o = o + torch.matmul(e_suf.reshape(kv_heads, seqs, q_len * group, most), v_suf.permute(2, 0, 1, 3)).view(kv_heads, seqs, q_len, group, dim)
    o = torch.where(total.unsqueeze(-1) > 0, o / total.unsqueeze(-1), 0.0)
    lse = base.squeeze(-1) + torch.log(total)
    live = (lens >= 0).view(-1, 1, 1)
    o = o.permute(1, 2, 0, 3, 4).reshape(seqs, q_len, heads, dim).to(state["out"].dtype)
    lse = lse.permute(1, 2, 0, 3).reshape(seqs, q_len, heads)
    state["out"].copy_(torch.where(live.unsqueeze(-1), o, state["out"]))
    state["lse"].copy_(torch.where(live, lse, state["lse"]))


def run(state):
    case = state["case"]
    if case["op"] == "write":
        if own:
            state["binding"].kv_cache_write_launch(state["handle"], state["key"], state["value"], state["slots"])
        else:
            _write_plain(state)
        if not case["readback"]:
            return dict(state["cache"])
    if case["op"] in ("write", "read"):
        if own:
            state["binding"].kv_cache_read_launch(state["handle"], state["slots"], state["key_out"], state["value_out"])
        else:
            live = state.get("live", case["tokens"])
            k, v = _read_plain(state["cache"], state["slots"][:live], state["key_out"].dtype)
            state["key_out"][:live], state["value_out"][:live] = k, v
        return {"key": state["key_out"], "value": state["value_out"]}
    if own:
        state["binding"].shared_prefix_attention_launch(state["handle"], state["batch"], state["q"], state["out"], state["lse"],
                                                        state["workspace"], softmax_scale=state["scale"])
    else:
        _attend_plain(state)
    return {"out": state["out"], "lse": state["lse"]}


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    held = size if case["fmt"] == "plain" else 1
    scale = 0 if case["fmt"] == "plain" else 4
    if case["op"] != "attend":
        vectors = 2 * case["tokens"] * case["kv_heads"]  # keys and values
        move = vectors * (case["dim"] * (size + held) + scale) + 8 * case["tokens"]
        passes = 2 if case["op"] == "write" and case["readback"] else 1
        return {"bytes": passes * move, "flops": passes * 2 * vectors * case["dim"]}
    lens = [n for n in _suffix_lengths(case) if n >= 0]
    q_len, heads, dim = case["q_len"], case["heads"], case["dim"]
    keys = case["prefix"] + sum(lens)
    rows = len(lens) * q_len * heads
    seen = sum(max(0, n - q_len + 1 + i) for n in lens for i in range(q_len)) * heads + rows * case["prefix"]
    return {"bytes": 2 * keys * case["kv_heads"] * (dim * held + scale) + rows * (2 * dim * size + 4), "flops": 4 * dim * seen}


# ---- 64 bits ----------------------------------------------------------------------------------------------------------

def _quantised64(x, fmt):
    """Codes and scales of binary64 vectors, the rounding to a code made by a search of the code values."""
    peak = torch.clamp(torch.amax(torch.abs(x), dim=-1, keepdim=True), min=1e-12)
    y = x / peak * CODE_MAX[fmt]
    if fmt == "int8":
        return torch.round(y), (peak / 127.0).squeeze(-1)
    # e4m3: steps of 2^(e-3) inside the binade e, and of 2^-9 below 2^-6
    e = torch.floor(torch.log2(torch.clamp(torch.abs(y), min=2.0 ** -6)))
    step = torch.pow(torch.full_like(e, 2.0), e - 3)
    return torch.round(y / step) * step, (peak / 448.0).squeeze(-1)


def exact(case, seed):
    state = prepare(case, seed)
    cache = {name: (t.float() if t.dtype != torch.float32 else t).double() for name, t in state["cache"].items()} if case["op"] != "attend" else state["cache"]
    if case["op"] == "write":
        live = state["live"]
        at = state["slots"][:live]
        back = {}
        for side, x in (("k", state["key"]), ("v", state["value"])):
            x = x[:live].double()
            values, scales = (x, None) if case["fmt"] == "plain" else _quantised64(x, case["fmt"])
            cache[side].view(-1, *cache[side].shape[2:])[at] = values
            if scales is not None:
                cache[side + "_scale"].view(-1, cache[side].shape[2])[at] = scales
            out = torch.zeros(case["tokens"], *x.shape[1:], dtype=torch.float64, device="cuda")
            out[:live] = values if scales is None else values * scales[..., None]
            back[{"k": "key", "v": "value"}[side]] = out
        return back if case["readback"] else cache
    if case["op"] == "read":
        got = {}
        for side, name in (("k", "key"), ("v", "value")):
            x = cache[side] if case["fmt"] == "plain" else cache[side] * cache[side + "_scale"][..., None]
            got[name] = x.reshape(-1, *x.shape[2:])[state["slots"]]
        return got
    q, lens = state["q"].double(), state["lens"].tolist()
    seqs, q_len, heads, dim = q.shape
    group = heads // case["kv_heads"]
    out = torch.zeros(seqs, q_len, heads, dim, dtype=torch.float64, device="cuda")
    lse = torch.zeros(seqs, q_len, heads, dtype=torch.float64, device="cuda")

    def entries(side, pages, n, head):
        x = cache[side][pages.long(), :, head].float().double().reshape(-1, dim)[:n]
        return x if case["fmt"] == "plain" else x * cache[side + "_scale"][pages.long(), :, head].double().reshape(-1, 1)[:n]

    for head in range(case["kv_heads"]):
        mine = slice(head * group, (head + 1) * group)
        k0, v0 = (entries(side, state["prefix_pages"], case["prefix"], head) for side in ("k", "v"))
        scores0 = (q[:, :, mine].reshape(-1, dim) @ k0.T * state["scale"])
        lse0 = torch.logsumexp(scores0, -1)
        out0 = (torch.exp(scores0 - lse0[:, None]) @ v0).view(seqs, q_len, group, dim)
        lse0 = lse0.view(seqs, q_len, group)
        for b, n in enumerate(lens):
            if n < 0:
                continue
            k1, v1 = (entries(side, state["page_table"][b], n, head) for side in ("k", "v"))
            scores1 = torch.einsum("qgd,kd->qgk", q[b, :, mine], k1) * state["scale"]
            hidden = torch.arange(n, device="cuda")[None, :] > (n - q_len + torch.arange(q_len, device="cuda"))[:, None]
            scores1 = scores1.masked_fill(hidden[:, None, :], float("-inf"))
            lse1 = torch.logsumexp(scores1, -1) if n else torch.full((q_len, group), float("-inf"), dtype=torch.float64, device="cuda")
            both = torch.logaddexp(lse0[b], lse1)
            lse[b, :, mine] = both
            own_part = torch.einsum("qgk,kd->qgd", torch.exp(scores1 - both[..., None]), v1)
            out[b, :, mine] = out0[b] * torch.exp(lse0[b] - both)[..., None] + own_part
    return {"out": out, "lse": lse}
