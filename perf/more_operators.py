"""Cases of three further serving operators: rotary positions, attention over packed prompts, and moving entries inside a
paged key/value cache (pages copied, tokens compacted).

``own`` is False: ``run`` computes the plain form (elementary torch operations in 32 bits, angles in 64).  Where it is True,
``run`` makes the calls of the package's binding that a serving program makes.

Rotary positions.  The first ``rot`` elements of a head are pairs (j, j + rot / 2), or (2 j, 2 j + 1) when interleaved.  Pair j
of a token at position p is turned by the angle p * theta_j and scaled by a magnitude:  y1 = m (x1 cos - x2 sin),
y2 = m (x2 cos + x1 sin); ``backward`` is the gradient, the opposite angle.  theta_j = base^(-2 j / rot), changed for long contexts: "linear"
theta_j / factor; "ntk" base * factor^(rot / (rot - 2)); "bands": with n_j = original * theta_j / 2 pi turns over the original
length, theta_j / factor below ``low`` turns, theta_j above ``high``, between them a line in n_j; "yarn": a line in j between the
whole numbers around the pairs of ``fast`` and ``slow`` turns, and m = 0.1 ln(factor) + 1.  A negative position is a padded token: its rows
stay as they were.

Prompt attention.  Sequences lie behind one another in [tokens, heads, dim] tensors; sequence b has the query rows
q_starts[b] .. q_starts[b + 1] and the key rows k_starts[b] .. k_starts[b + 1].  Causal: query i of n_q sees the keys j <= n_k - n_q + i.
Query head h reads key/value head h // (heads / kv_heads).  Outputs: the result and the natural logarithm of the softmax
denominator (a zero row and -inf where no key is seen); rows behind the last sequence stay as they were.

Pages.  A cache of several layers.  Copy: the first tokens of page src[i] become those of page dst[i] in every layer.  Compact: of the tokens
starts[b] .. lens[b] of a sequence those with keep[b, i] move to starts[b], starts[b] + 1, ... in their order.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
CODE_TYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
SCORES = 1 << 30  # scores that the plain form holds at a time


def _rotary(name, tokens, heads, kv_heads, dim, rot, dtype, interleaved=False, scaling="none", far=4096, backward=False, padded=0):
    return {"name": name, "op": "rotary", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rot": rot, "dtype": dtype,
            "interleaved": interleaved, "scaling": scaling, "far": far, "backward": backward, "padded": padded}


def _prompt(name, seqs, longest, heads, kv_heads, dim, dtype, context=0, ragged=False, causal=True, tail=0):
    return {"name": name, "op": "prompt", "seqs": seqs, "longest": longest, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
            "context": context, "ragged": ragged, "causal": causal, "tail": tail}


def _copy(name, layers, copied, page, heads, dim, fmt, partial):
    return {"name": name, "op": "copy", "layers": layers, "copied": copied, "page": page, "kv_heads": heads, "dim": dim, "fmt": fmt, "partial": partial}


def _compact(name, layers, seqs, before, window, page, heads, dim, fmt, kept, padded=0):
    return {"name": name, "op": "compact", "layers": layers, "seqs": seqs, "before": before, "window": window, "page": page, "kv_heads": heads,
            "dim": dim, "fmt": fmt, "kept": kept, "padded": padded}


def listed():
    return [
        # the queries and keys of one decoding step of a batch of 64: latency counts
        _rotary("rotary_64x32of8x128_bf16", 64, 32, 8, 128, 128, "bf16", far=32768),
        # a prefill of 16384 tokens on a context that was stretched eightfold
        _rotary("rotary_16384x32of8x128_bf16_yarn", 16384, 32, 8, 128, 128, "bf16", scaling="yarn", far=65536),
        # the gradient for heads whose last elements are not turned, pairs side by side, odd sizes, far positions
        _rotary("rotary_1001x5of5x80_fp16_back", 1001, 5, 5, 80, 64, "fp16", True, "bands", 1 << 20, True, 17),
        # one short question: latency counts
        _prompt("prompt_1x100_32of8x128", 1, 100, 32, 8, 128, "bf16"),
        # a batch of prompts of all lengths from none to 1500 tokens, heads of 64, padded to a fixed number of rows
        _prompt("prompt_17x1500_8of8x64_ragged_fp16", 17, 1500, 8, 8, 64, "fp16", ragged=True, tail=100),
        # a chunk of 512 tokens of a long prompt behind 16000 tokens that were fetched out of the cache; five query heads per key/value head
        _prompt("prompt_1x512_40of8x128_behind_16000", 1, 512, 40, 8, 128, "bf16", context=16000),
        # heads of 256
        _prompt("prompt_4x2000_32of4x256_ragged", 4, 2000, 32, 4, 256, "bf16", ragged=True),
        # a document of 16384 tokens
        _prompt("prompt_1x16384_32of8x128", 1, 16384, 32, 8, 128, "bf16"),
        # three continuations of a few conversations: their last, partly filled pages copied
        _copy("copy_12_pages_of_16x8x128_32_layers", 32, 12, 16, 8, 128, "bf16", True),
        # a cache rearranged: 512 pages of every layer
        _copy("copy_500_pages_of_64x8x128_e4m3_16_layers", 16, 500, 64, 8, 128, "e4m3", False),
        # the accepted ones of seven drafted tokens of every sequence
        _compact("compact_40x7_32_layers_8x128", 32, 40, 200, 7, 16, 8, 128, "bf16", 0.4, 3),
        # half of each context given up
        _compact("compact_12x4000_int8_8_layers_8x128", 8, 12, 4, 4000, 32, 8, 128, "int8", 0.5),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["rotary", "prompt", "prompt", "copy", "compact"])
    if op == "rotary":
        kv_heads, group, dim = rng.choice([1, 2, 4, 5, 8]), rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 80, 96, 128, 128, 256])
        rot = rng.choice([dim, dim, dim // 2, 32, 48])
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        most = 16384 * 40 * 128 // (2 if dtype == "fp32" else 1)
        tokens = _log_uniform(rng, 1, min(16384, most // ((group + 1) * kv_heads * dim)))
        case = _rotary("", tokens, group * kv_heads, kv_heads, dim, rot, dtype, rng.random() < 0.4, rng.choice(["none", "linear", "ntk", "bands", "yarn"]),
                       _log_uniform(rng, 16, 1 << 20), rng.random() < 0.3, rng.choice([0, tokens // 7]))
    elif op == "prompt":
        kv_heads, group, dim = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 64, 80, 96, 128, 128, 128, 256])
        seqs, longest = _log_uniform(rng, 1, 128), _log_uniform(rng, 1, 16384)
        context = rng.choice([0, 0, 0, _log_uniform(rng, 1, 16384)])
        group = min(group, max(1, 32 // kv_heads))
        while (seqs * longest * (longest + context) * kv_heads * group * dim > 32 * 128 * 16384 * 16384 // 2
               or seqs * (longest + context) * kv_heads * (group + 2) * dim > 4 * 16384 * 48 * 128):
            if seqs > 1:
                seqs = max(1, seqs // 2)
            else:
                longest, context = max(1, longest // 2), context // 2
        case = _prompt("", seqs, longest, kv_heads * group, kv_heads, dim, rng.choice(["bf16", "bf16", "fp16"]), context, rng.random() < 0.6, rng.random() < 0.85,
                       rng.choice([0, 0, 33]))
    else:
        heads, dim, page, fmt = rng.choice([1, 2, 4, 5, 8]), rng.choice([33, 64, 80, 128, 128, 256]), rng.choice([1, 8, 16, 32, 64]), rng.choice(["bf16", "bf16", "e4m3", "int8"])
        layers = rng.choice([1, 4, 12, 32])
        size = 2 if fmt == "bf16" else 1
        most = 16 * 500 * 64 * 8 * 128 // (layers * heads * dim * size)  # tokens
        if op == "copy":
            case = _copy("", layers, _log_uniform(rng, 1, max(1, min(2000, most // page))), page, heads, dim, fmt, rng.random() < 0.5)
        else:
            window = _log_uniform(rng, 1, 4000)
            seqs = _log_uniform(rng, 1, max(1, min(64, most // (window + 64))))
            case = _compact("", layers, seqs, _log_uniform(rng, 1, 200), min(window, max(1, most)), page, heads, dim, fmt, rng.choice([0.1, 0.5, 0.9]), rng.choice([0, seqs // 5]))
    del case["name"]
    return case


# ---- inputs -------------------------------------------------------------------------------------------------------

def _spec(case):
    """How the frequencies are scaled: a base and the numbers of the scaling."""
    return {"none": dict(base=10000.0, factor=1.0), "linear": dict(base=10000.0, factor=4.0), "ntk": dict(base=10000.0, factor=8.0),
            "bands": dict(base=500000.0, factor=8.0, original=8192, low=1.0, high=4.0),
            "yarn": dict(base=1000000.0, factor=8.0, original=8192, fast=32.0, slow=1.0)}[case["scaling"]]


def _frequencies(case):
    """(theta_j in binary64 on the GPU, magnitude)."""
    p, rot, kind = _spec(case), case["rot"], case["scaling"]
    j = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    base = p["base"] * p["factor"] ** (rot / (rot - 2)) if kind == "ntk" else p["base"]
    theta = torch.exp(j * (-2.0 * math.log(base) / rot))
    if kind == "linear":
        theta = theta / p["factor"]
    if kind == "bands":
        line = ((p["original"] * theta / (2 * math.pi) - p["low"]) / (p["high"] - p["low"])).clamp(0, 1)
        theta = theta * line + theta / p["factor"] * (1 - line)
    if kind == "yarn":
        pair = lambda turns: rot * math.log(p["original"] / (2 * math.pi * turns)) / (2 * math.log(base))
        first, last = max(0, math.floor(pair(p["fast"]))), min(rot - 1, math.ceil(pair(p["slow"])))
        line = ((j - first) / max(last - first, 0.001)).clamp(0, 1)
        theta = theta / p["factor"] * line + theta * (1 - line)
    return theta, 0.1 * math.log(p["factor"]) + 1 if kind == "yarn" else 1.0


def _lengths(case):
    """[(query tokens, keys)] of the sequences, before they are shuffled."""
    n = case["seqs"]
    q = [case["longest"]] * n if not case["ragged"] else [round(case["longest"] * (i + 1) / n) for i in range(n)]
    if case["ragged"] and n > 2:
        q[0] = 0  # an empty place of the batch
    return [(a, a + case["context"] * (n - i) // n) for i, a in enumerate(q)]


def _fill(shape, dtype, gen):
    """Values as projections make them: channels of different strengths, a few of them strong."""
    channel = torch.exp(0.4 * torch.randn(shape[-2:], generator=gen, device="cuda"))
    return (torch.randn(shape, generator=gen, device="cuda") * channel).to(dtype)


def _new_layers(case, n_pages, gen):
    """Keys and values of all layers as one tensor [layers, 2, pages, page, heads, dim], and their scales."""
    shape = (case["layers"], 2, n_pages, case["page"], case["kv_heads"], case["dim"])
    if case["fmt"] == "bf16":
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16), None
    if case["fmt"] == "e4m3":  # every code but the two of a NaN
        codes = torch.randint(0, 254, shape, generator=gen, device="cuda", dtype=torch.uint8)
        codes = codes.add_(codes >= 127).view(torch.float8_e4m3fn)
    else:
        codes = torch.randint(-127, 128, shape, generator=gen, device="cuda", dtype=torch.int8)
    return codes, torch.rand(shape[:-1], generator=gen, device="cuda") + 0.01


def _prepare_pages(case, gen, state):
    page = case["page"]
    if case["op"] == "copy":
        n = case["copied"]
        n_pages = 2 * n + 3
        order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        state["dst"] = order[:n].contiguous()
        # a page out of three is copied more than once
        state["src"] = order[n:][torch.randint(0, max(1, 2 * n // 3), (n,), generator=gen, device="cuda")].contiguous()
        state["tokens"] = torch.randint(1, page + 1, (n,), generator=gen, device="cuda", dtype=torch.int32) if case["partial"] else None
    else:
        seqs, window = case["seqs"], case["window"]
        live = seqs - case["padded"]
        starts = torch.randint(0, case["before"] + 1, (seqs,), generator=gen, device="cuda", dtype=torch.int32)
        used = torch.randint((window + 1) // 2, window + 1, (seqs,), generator=gen, device="cuda", dtype=torch.int32)
        lens = starts + used
        lens[live:] = -1
        per_seq = (lens.clamp_min(0) + page - 1) // page
        width = -(-(case["before"] + window) // page)
        n_pages = seqs * width + 2
        order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        begin = torch.cumsum(per_seq, 0) - per_seq
        column = torch.arange(width, device="cuda")
        state["table"] = torch.where(column < per_seq.unsqueeze(1), order[(begin.unsqueeze(1) + column).clamp_max(n_pages - 1).long()], 0).to(torch.int32)
        state["starts"], state["lens"] = starts, lens
        state["keep"] = torch.rand(seqs, window, generator=gen, device="cuda") < case["kept"]
        state["new_lens"] = torch.zeros(seqs, device="cuda", dtype=torch.int32)
    state["kv"], state["scale"] = _new_layers(case, n_pages, gen)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = {"case": dict(case)}
    if case["op"] == "rotary":
        tokens, heads, kv_heads, dim, dtype = case["tokens"], case["heads"], case["kv_heads"], case["dim"], DTYPES[case["dtype"]]
        # queries and keys as they leave the projection: slices of one [tokens, heads + 2 * kv_heads, dim] tensor
        both = _fill((tokens, heads + 2 * kv_heads, dim), dtype, gen)
        state["q"], state["k"] = both[:, :heads], both[:, heads:heads + kv_heads]
        state["q_out"] = torch.zeros(tokens, heads, dim, dtype=dtype, device="cuda")
        state["k_out"] = torch.zeros(tokens, kv_heads, dim, dtype=dtype, device="cuda")
        state["positions"] = torch.randint(0, case["far"], (tokens,), generator=gen, device="cuda")
        if case["padded"]:
            state["positions"][tokens - case["padded"]:] = -1
        state["live"] = tokens - case["padded"]
        if own:
            from paper_2601_12698_b200 import binding
            p = _spec(case)
            names = {"original": "original_len", "low": "low_turns", "high": "high_turns", "fast": "fast_turns", "slow": "slow_turns"}
            state["binding"] = binding
            state["table"] = binding.RotaryTable(case["rot"], scaling=case["scaling"], interleaved=case["interleaved"],
                                                 **{names.get(k, k): v for k, v in p.items()})
        else:
            state["theta"], state["magnitude"] = _frequencies(case)
    elif case["op"] == "prompt":
        lens = _lengths(case)
        order = torch.randperm(len(lens), generator=gen, device="cuda").tolist()
        lens = [lens[i] for i in order]
        q_lens, k_lens = (torch.tensor(x, device="cuda", dtype=torch.int32) for x in zip(*lens))
        zero = torch.zeros(1, device="cuda", dtype=torch.int32)
        state["q_starts"], state["k_starts"] = (torch.cat([zero, torch.cumsum(x, 0).to(torch.int32)]) for x in (q_lens, k_lens))
        dtype, dim = DTYPES[case["dtype"]], case["dim"]
        rows, keys = sum(a for a, _ in lens) + case["tail"], sum(b for _, b in lens) + case["tail"]
        state["q"] = torch.randn(rows, case["heads"], dim, generator=gen, device="cuda").to(dtype)
        both = _fill((keys, 2 * case["kv_heads"], dim), dtype, gen)
        state["k"], state["v"] = both[:, :case["kv_heads"]], both[:, case["kv_heads"]:]
        state["out"] = torch.zeros_like(state["q"])
        state["lse"] = torch.zeros(rows, case["heads"], dtype=torch.float32, device="cuda")
        state["scale"] = 1.0 / math.sqrt(dim)
        state["longest"] = (max(a for a, _ in lens), max(b for _, b in lens))
        if own:
            from paper_2601_12698_b200 import binding
            state["binding"] = binding
            state["batch"] = binding.PromptBatch(state["q_starts"], state["longest"][0], state["k_starts"], state["longest"][1], causal=case["causal"])
            state["workspace"] = binding.prompt_attention_workspace(state["batch"], state["q"], state["k"])
    else:
        _prepare_pages(case, gen, state)
        if own:
            from paper_2601_12698_b200 import binding
            kv, scale = state["kv"], state["scale"]
            state["binding"] = binding
            state["stack"] = binding.KvCacheStack([binding.KvCache(kv[l, 0], kv[l, 1], *(() if scale is None else (scale[l, 0], scale[l, 1])))
                                                   for l in range(case["layers"])])
    return state


# ---- the passes -----------------------------------------------------------------------------------------------------

def _rotary_plain(state):
    case, live, rot = state["case"], state["live"], state["case"]["rot"]
    angle = state["positions"][:live].double().unsqueeze(1) * state["theta"]
    cos, sin = ((f(angle) * state["magnitude"]).float().unsqueeze(1) for f in (torch.cos, torch.sin))
    if case["backward"]:
        sin = -sin
    for x, out in ((state["q"], state["q_out"]), (state["k"], state["k_out"])):
        x, out = x[:live].float(), out[:live]
        if case["interleaved"]:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        else:
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        pair = (a * cos - b * sin, b * cos + a * sin)
        turned = torch.stack(pair, -1).flatten(-2) if case["interleaved"] else torch.cat(pair, -1)
        out.copy_(torch.cat([turned, x[..., rot:]], -1))


def _prompt_plain(state):
    """The sequences side by side in a padded batch; some of its rows at a time."""
    case, out, lse = state["case"], state["out"], state["lse"]
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    group = heads // kv_heads
    (q_from, q_to), (k_from, k_to) = ((s[:-1].long(), s[1:].long()) for s in (state["q_starts"], state["k_starts"]))
    n_q, n_k = q_to - q_from, k_to - k_from
    most_q, most_k = state["longest"]
    key_at = torch.arange(most_k, device="cuda")
    key_rows = (k_from.unsqueeze(1) + key_at).clamp_max(max(0, state["k"].shape[0] - 1))
    there = key_at < n_k.unsqueeze(1)                                                                    # [B, keys]
    k = state["k"][key_rows].float().permute(0, 2, 3, 1)                                                 # [B, K, d, keys]
    v = state["v"][key_rows].float().masked_fill(~there[..., None, None], 0.0).permute(0, 2, 1, 3)       # [B, K, keys, d]
    step = max(1, SCORES // max(1, case["seqs"] * heads * most_k))
    for first in range(0, most_q, step):
        at = torch.arange(first, min(first + step, most_q), device="cuda")
        mine = at < n_q.unsqueeze(1)                                                                     # [B, rows]
        rows = (q_from.unsqueeze(1) + at).clamp_max(state["q"].shape[0] - 1)
        q = state["q"][rows].float().view(case["seqs"], at.numel(), kv_heads, group, dim).permute(0, 2, 3, 1, 4) * state["scale"]
        s = torch.matmul(q.reshape(case["seqs"], kv_heads, -1, dim), k).view(case["seqs"], kv_heads, group, at.numel(), most_k)
        seen = there.unsqueeze(1)
        if case["causal"]:
            seen = seen & (key_at <= (n_k - n_q).view(-1, 1, 1) + at.unsqueeze(1))                       # [B, rows, keys]
        s.masked_fill_(~seen[:, None, None], float("-inf"))
        top = s.amax(-1, keepdim=True)
        top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
        s = s.sub_(top).exp_()
        total = s.sum(-1)
        o = torch.matmul(s.view(case["seqs"], kv_heads, -1, most_k), v).view(case["seqs"], kv_heads, group, at.numel(), dim)
        o = torch.where(total.unsqueeze(-1) > 0, o / total.unsqueeze(-1), 0.0)
        got = top.squeeze(-1) + torch.log(total)
        out[rows[mine]] = o.permute(0, 3, 1, 2, 4).reshape(case["seqs"], at.numel(), heads, dim)[mine].to(out.dtype)
        lse[rows[mine]] = got.permute(0, 3, 1, 2).reshape(case["seqs"], at.numel(), heads)[mine]


def _move_plain(state, src, dst):
    """Entries of the slots `src` to the slots `dst`, in all layers."""
    for t in (state["kv"], state["scale"]):
        if t is not None:
            flat = (t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t).flatten(2, 3)
            flat[:, :, dst] = flat[:, :, src]


def _copy_plain(state):
    page = state["case"]["page"]
    at = torch.arange(page, device="cuda")
    src, dst = (x.long().unsqueeze(1) * page + at for x in (state["src"], state["dst"]))
    if state["tokens"] is not None:
        some = at < state["tokens"].unsqueeze(1)
        src, dst = src[some], dst[some]
    _move_plain(state, src.flatten(), dst.flatten())


def _compact_plain(state):
    page, lens, starts = state["case"]["page"], state["lens"].long(), state["starts"].long()
    at = torch.arange(state["case"]["window"], device="cuda")
    keep = state["keep"] & (at < (lens - starts).unsqueeze(1))
    to = torch.cumsum(keep, 1) - 1
    slot = lambda pos: torch.gather(state["table"].long(), 1, (pos // page).clamp(0, state["table"].shape[1] - 1)) * page + pos % page
    src, dst = slot(starts.unsqueeze(1) + at), slot(starts.unsqueeze(1) + to.clamp_min(0))
    _move_plain(state, src[keep], dst[keep])
    state["new_lens"].copy_(torch.where(lens < 0, lens, starts + keep.sum(1)))


def run(state):
    case, op = state["case"], state["case"]["op"]
    if op == "rotary":
        if own:
            state["binding"].rotary_launch(state["table"], state["positions"], state["q"], state["k"], state["q_out"], state["k_out"], backward=case["backward"])
        else:
            _rotary_plain(state)
        return {"q": state["q_out"], "k": state["k_out"]}
    if op == "prompt":
        if own:
            state["binding"].prompt_attention_launch(state["batch"], state["q"], state["k"], state["v"], state["out"], state["lse"], state["workspace"],
                                                     softmax_scale=state["scale"])
        else:
            _prompt_plain(state)
        return {"out": state["out"], "lse": state["lse"]}
    if op == "copy":
        if own:
            state["binding"].kv_cache_copy_pages_launch(state["stack"], state["src"], state["dst"], state["tokens"])
        else:
            _copy_plain(state)
        return {"kv": state["kv"], "scale": state["scale"]}
    if own:
        state["binding"].kv_cache_compact_launch(state["stack"], state["table"], state["starts"], state["lens"], state["keep"], state["new_lens"])
    else:
        _compact_plain(state)
    return {"kv": state["kv"], "scale": state["scale"], "new_lens": state["new_lens"]}


def work(case):
    op = case["op"]
    if op == "rotary":
        live, size = case["tokens"] - case["padded"], 4 if case["dtype"] == "fp32" else 2
        heads = case["heads"] + case["kv_heads"]
        return {"bytes": live * heads * case["dim"] * 2 * size + 8 * case["tokens"], "flops": live * heads * case["rot"] * 3}
    if op == "prompt":
        lens = _lengths(case)
        seen = sum(sum(max(0, n_k - n_q + 1 + i) for i in range(n_q)) if case["causal"] else n_q * n_k for n_q, n_k in lens)
        rows, keys = sum(a for a, _ in lens), sum(b for _, b in lens)
        return {"bytes": rows * case["heads"] * (4 * case["dim"] + 4) + 4 * keys * case["kv_heads"] * case["dim"], "flops": 4 * case["dim"] * case["heads"] * seen}
    entry = case["dim"] * 2 if case["fmt"] == "bf16" else case["dim"] + 4
    if op == "copy":
        tokens = case["copied"] * (case["page"] + 1) // 2 if case["partial"] else case["copied"] * case["page"]
    else:  # the kept tokens of a window that is three quarters full on average; those before the first gap stay
        tokens = max(1, int((case["seqs"] - case["padded"]) * case["window"] * 0.75 * case["kept"]))
    return {"bytes": 2 * 2 * case["layers"] * tokens * case["kv_heads"] * entry, "flops": 0}


# ---- 64 bits ----------------------------------------------------------------------------------------------------------

def exact(case, seed):
    """Copies and compactions compute nothing: their outputs are compared with the plain form's alone."""
    if case["op"] in ("copy", "compact"):
        return None
    state = prepare(case, seed)
    if case["op"] == "rotary":
        theta, magnitude = (state["theta"], state["magnitude"]) if "theta" in state else _frequencies(case)
        live, rot = state["live"], case["rot"]
        # complex numbers: a pair is one, a turn a product
        turn = torch.polar(torch.full((live, rot // 2), magnitude, dtype=torch.float64, device="cuda"),
                           (-1 if case["backward"] else 1) * torch.outer(state["positions"][:live].double(), theta))
        got = {}
        for name in ("q", "k"):
            x = state[name].double()
            y = torch.zeros_like(x, memory_format=torch.contiguous_format)
            y[:live, :, rot:] = x[:live, :, rot:]
            index = torch.arange(rot, device="cuda")
            first, second = (index[0::2], index[1::2]) if case["interleaved"] else (index[:rot // 2], index[rot // 2:])
            z = torch.complex(x[:live][..., first], x[:live][..., second]) * turn[:, None]
            y[:live, :, first], y[:live, :, second] = z.real, z.imag
            got[name] = y
        return got
    heads, dim = case["heads"], case["dim"]
    group = heads // case["kv_heads"]
    out = torch.zeros(*state["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(*state["lse"].shape, dtype=torch.float64, device="cuda")
    q_starts, k_starts = state["q_starts"].tolist(), state["k_starts"].tolist()
    for b in range(case["seqs"]):
        n_q, n_k = q_starts[b + 1] - q_starts[b], k_starts[b + 1] - k_starts[b]
        for head in range(case["kv_heads"]):
            k, v = (state[x][k_starts[b]:k_starts[b + 1], head].double() for x in ("k", "v"))
            for first in range(0, n_q, 1024):
                last = min(first + 1024, n_q)
                rows, mine = slice(q_starts[b] + first, q_starts[b] + last), slice(head * group, (head + 1) * group)
                sees = n_k - n_q + last if case["causal"] else n_k
                s = torch.einsum("igd,jd->igj", state["q"][rows, mine].double(), k[:sees]) * state["scale"]
                if case["causal"]:
                    i, j = torch.arange(first, last, device="cuda"), torch.arange(sees, device="cuda")
                    s = s.masked_fill((j[None, :] > (n_k - n_q + i)[:, None])[:, None, :], float("-inf"))
                total = torch.logsumexp(s, -1)
                lse[rows, mine] = total
                out[rows, mine] = torch.einsum("igj,jd->igd", torch.exp(s - total[..., None]), v[:sees])
    return {"out": out, "lse": lse}
