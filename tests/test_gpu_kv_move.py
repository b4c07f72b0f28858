"""Pages copied and gaps closed inside caches, bit for bit against indexing on the CPU, and what must stay untouched."""
import pytest
import torch

from test_gpu_kv_cache import B, TD, _as, _cache  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu


def _stack(B, layers, layout, pages, page, heads, dim, dtype, fmt, seed=0):
    """A stack of caches filled with random bytes; (stack, their base tensors)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    caches, bases = [], []
    for _ in range(layers):
        cache, base = _cache(B, layout, pages, page, heads, dim, dtype, fmt)
        for t in base:
            flat = t.view(torch.uint8) if t.dtype != torch.uint8 else t
            flat.copy_(torch.randint(0, 256, flat.shape, generator=g, device="cuda", dtype=torch.uint8))
        for t in (cache.k_scale, cache.v_scale):
            if t is not None:
                t.copy_(torch.rand(t.shape, generator=g, device="cuda"))
        caches.append(cache)
        bases.append(base)
    return B.KvCacheStack(caches), bases


def _bytes(t):
    """Entries [pages, page, heads, bytes] of a cache's tensor on the CPU."""
    t = t.cpu() if t.dtype != torch.float8_e4m3fn else t.view(torch.uint8).cpu()
    if t.dim() == 3:
        t = t.unsqueeze(-1)
    return t.contiguous().view(torch.uint8).reshape(*t.shape[:3], -1)


def _sides(stack):
    return [t for c in stack.caches for t in (c.k, c.v, c.k_scale, c.v_scale) if t is not None]


def _gaps(bases):
    """What lies between the entries of a layout with gaps."""
    return [t[..., -16:].contiguous().view(torch.uint8).cpu() for base in bases for t in base if t.dim() == 5]


SHAPES = [(1, "token", 16, 8, 128, "bf16", "plain"), (3, "head", 16, 5, 100, "fp16", "int8"), (2, "gap", 8, 2, 64, "bf16", "e4m3"), (2, "token", 1, 3, 33, "bf16", "int8"),
          (1, "head", 24, 4, 33, "fp32", "plain"), (2, "gap", 7, 3, 80, "fp32", "plain"), (4, "token", 64, 8, 128, "bf16", "e4m3"), (1, "token", 32, 1, 256, "fp16", "plain"),
          (1, "token", 16, 1, 1, "bf16", "int8"), (2, "token", 5, 2, 3, "bf16", "plain"), (1, "token", 200, 8, 256, "fp32", "plain")]


@pytest.mark.parametrize("layers,layout,page,heads,dim,dtype,fmt", SHAPES)
@pytest.mark.parametrize("n,partial", [(1, False), (9, True), (70, False), (33, True)])
def test_pages_are_copied(B, layers, layout, page, heads, dim, dtype, fmt, n, partial):
    pages = 2 * n + 4
    stack, bases = _stack(B, layers, layout, pages, page, heads, dim, dtype, fmt, n)
    g = torch.Generator().manual_seed(n)
    order = torch.randperm(pages, generator=g).int()
    src, dst = order[n:][torch.randint(0, n, (n,), generator=g)], order[:n].clone()
    tokens = torch.randint(0, page + 1, (n,), generator=g).int() if partial else None
    if n > 8:
        src[3] = -1
        dst[5] = -4
    want = [_bytes(t) for t in _sides(stack)]
    gaps = _gaps(bases)
    for w in want:
        old = w.clone()
        for i in range(n):
            if src[i] >= 0 and dst[i] >= 0:
                some = page if tokens is None else int(tokens[i])
                w[dst[i], :some] = old[src[i], :some]
    B.kv_cache_copy_pages_launch(stack, src.cuda(), dst.cuda(), None if tokens is None else tokens.cuda())
    for t, w in zip(_sides(stack), want):
        assert torch.equal(_bytes(t), w)
    assert all(torch.equal(a, b) for a, b in zip(gaps, _gaps(bases)))
    assert B.rt_device_status() == 0


def test_pages_and_lengths_outside_are_skipped_and_reported(B):
    stack, _ = _stack(B, 2, "token", 8, 4, 2, 16, "bf16", "int8")
    want = [_bytes(t) for t in _sides(stack)]
    for w in want:
        w[4] = w[0]       # tokens cut to a page
        w[6, :0] = w[1, :0]
    src, dst, tokens = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 8, 1, 2, 1], [4, 5, 100, 1 << 30, 6], [9, 4, 4, 4, -3]))
    B.kv_cache_copy_pages_launch(stack, src, dst, tokens)
    assert B.rt_device_status() == B.RT_ERR_INDEX
    for t, w in zip(_sides(stack), want):
        assert torch.equal(_bytes(t), w)


def _compact_reference(want, table, starts, lens, keep, page):
    """The moves on the entries, a token at a time; returns the new lengths."""
    new = []
    for b in range(len(lens)):
        start, n = int(starts[b]), int(lens[b])
        if n < 0:
            new.append(n)
            continue
        at = start
        for i in range(n - start):
            if keep[b, i]:
                for w in want:
                    w[table[b, at // page], at % page] = w[table[b, (start + i) // page], (start + i) % page]
                at += 1
        new.append(at)
    return new


def _check_moves(stack, want, table, lens, new, page):
    """Entries up to the new lengths, and everything that belongs to no sequence's tail."""
    loose = torch.zeros(want[0].shape[:2], dtype=torch.bool)
    for b in range(len(lens)):
        for at in range(max(new[b], 0), max(int(lens[b]), 0)):
            loose[table[b, at // page], at % page] = True
    for t, w in zip(_sides(stack), want):
        assert torch.equal(_bytes(t)[~loose], w[~loose])


@pytest.mark.parametrize("layers,layout,page,heads,dim,dtype,fmt", SHAPES)
@pytest.mark.parametrize("seqs,window,kept", [(1, 1, 0.5), (5, 7, 0.4), (3, 300, 0.5), (2, 700, 0.97), (4, 64, 0.0), (2, 260, 1.0)])
def test_gaps_are_closed(B, layers, layout, page, heads, dim, dtype, fmt, seqs, window, kept):
    g = torch.Generator().manual_seed(window + seqs)
    starts = torch.randint(0, 40, (seqs,), generator=g).int()
    lens = starts + torch.randint(window // 2, window + 1, (seqs,), generator=g).int()
    if seqs > 3:
        lens[2] = -1
    width = -(-(40 + window) // page)
    pages = seqs * width + 2
    table = torch.randperm(pages, generator=g).int()[:seqs * width].reshape(seqs, width)
    keep = torch.rand(seqs, window, generator=g) < kept
    stack, bases = _stack(B, layers, layout, pages, page, heads, dim, dtype, fmt, seqs)
    want, gaps = [_bytes(t) for t in _sides(stack)], _gaps(bases)
    new = _compact_reference(want, table, starts, lens, keep, page)
    got = torch.full((seqs,), -9, dtype=torch.int32, device="cuda")
    wide = torch.zeros(seqs, window + 5, dtype=torch.bool, device="cuda")  # rows with a stride of their own
    wide[:, :window] = keep.cuda()
    B.kv_cache_compact_launch(stack, table.cuda(), starts.cuda(), lens.cuda(), wide[:, :window], got)
    assert got.tolist() == new
    _check_moves(stack, want, table, lens, new, page)
    assert all(torch.equal(a, b) for a, b in zip(gaps, _gaps(bases)))
    assert B.rt_device_status() == 0


@pytest.mark.parametrize("layers,layout,page,heads,dim,dtype,fmt", SHAPES)
def test_gaps_are_closed_in_long_windows(B, layers, layout, page, heads, dim, dtype, fmt):
    """Windows of several thousand tokens, which go by in pieces."""
    test_gaps_are_closed(B, layers, layout, page, heads, dim, dtype, fmt, 2, 2600, 0.7)


def test_a_wide_layer_stack_is_compacted_by_many_ctas(B):
    stack, _ = _stack(B, 40, "token", 30, 16, 8, 128, "bf16", "int8")
    g = torch.Generator().manual_seed(5)
    table = torch.randperm(30, generator=g).int()[:28].reshape(7, 4)
    starts, lens = torch.full((7,), 20).int(), torch.randint(20, 60, (7,), generator=g).int()
    keep = torch.rand(7, 40, generator=g) < 0.5
    want = [_bytes(t) for t in _sides(stack)]
    new = _compact_reference(want, table, starts, lens, keep, 16)
    got = torch.zeros(7, dtype=torch.int32, device="cuda")
    B.kv_cache_compact_launch(stack, table.cuda(), starts.cuda(), lens.cuda(), keep.to(torch.uint8).cuda(), got)
    assert got.tolist() == new
    _check_moves(stack, want, table, lens, new, 16)


def test_sequences_that_do_not_fit_are_left_and_reported(B):
    stack, _ = _stack(B, 1, "token", 12, 4, 2, 16, "bf16", "plain")
    before = [_bytes(t) for t in _sides(stack)]
    table = torch.arange(12, dtype=torch.int32).reshape(4, 3).cuda()
    starts = torch.tensor([0, -1, 5, 2], dtype=torch.int32, device="cuda")
    lens = torch.tensor([9, 3, 4, 13], dtype=torch.int32, device="cuda")  # longer than the window, below zero, behind its end, longer than its pages
    keep, new = torch.zeros(4, 8, dtype=torch.bool, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    keep[:, 1::2] = True
    B.kv_cache_compact_launch(stack, table, starts, lens, keep, new)
    assert B.rt_device_status() == B.RT_ERR_INDEX and new.tolist() == lens.tolist()
    assert all(torch.equal(_bytes(t), w) for t, w in zip(_sides(stack), before))
    # a page outside the cache: its tokens are not moved, the others are
    table[0, 1] = 99
    starts, lens = torch.tensor([0, 0, 0, 0], dtype=torch.int32, device="cuda"), torch.tensor([8, -1, -1, -1], dtype=torch.int32, device="cuda")
    want = [w.clone() for w in before]
    for w in want:
        w[0, 0], w[0, 1] = before[0][0, 1] if w is want[0] else before[1][0, 1], before[0][0, 3] if w is want[0] else before[1][0, 3]
    B.kv_cache_compact_launch(stack, table, starts, lens, keep, new)
    assert B.rt_device_status() == B.RT_ERR_INDEX and new.tolist() == [4, -1, -1, -1]
    for t, w in zip(_sides(stack), want):
        assert torch.equal(_bytes(t)[0, :2], w[0, :2]) and torch.equal(_bytes(t)[3:], w[3:])


def test_streams_graphs_and_refusals(B):
    stack, _ = _stack(B, 2, "token", 20, 16, 4, 64, "bf16", "e4m3")
    src, dst = torch.arange(5, dtype=torch.int32, device="cuda"), torch.arange(10, 15, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.kv_cache_copy_pages_launch(stack, src, dst)
    src += 5
    graph.replay()
    for t in _sides(stack):
        assert torch.equal(_bytes(t)[10:15], _bytes(t)[5:10])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.kv_cache_copy_pages_launch(stack, src - 5, dst, stream=side)
    side.synchronize()
    for t in _sides(stack):
        assert torch.equal(_bytes(t)[10:15], _bytes(t)[:5])
    B.kv_cache_copy_pages_launch(stack, src[:0], dst[:0])
    for bad in (dict(src=src.long()), dict(dst=dst[:3]), dict(src=src.cpu()), dict(tokens=src[:2]), dict(dst=dst.float())):
        with pytest.raises(ValueError):
            B.kv_cache_copy_pages_launch(stack, **{**dict(src=src, dst=dst), **bad})
    lens, keep = torch.full((2,), 30, dtype=torch.int32, device="cuda"), torch.ones(2, 8, dtype=torch.bool, device="cuda")
    table, starts, new = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), lens - 4, torch.empty_like(lens)
    for bad in (dict(lens=lens[:1]), dict(keep=keep.float()), dict(keep=keep[:1]), dict(table=table.long()), dict(table=table[:1]), dict(new=new.long()), dict(keep=keep.t())):
        args = {**dict(table=table, starts=starts, lens=lens, keep=keep, new=new), **bad}
        with pytest.raises(ValueError):
            B.kv_cache_compact_launch(stack, args["table"], args["starts"], args["lens"], args["keep"], args["new"])
    with pytest.raises(B.TunerError):
        B.kv_cache_compact_launch(stack, table, starts, lens, keep, lens)
    with pytest.raises(ValueError):
        B.KvCacheStack([])
    with pytest.raises(ValueError):
        B.KvCacheStack([stack.caches[0], B.KvCache.allocate(20, 8, 4, 64, torch.float8_e4m3fn)])


def test_a_stack_holds_no_cache_twice(B):
    cache = B.KvCache.allocate(4, 8, 2, 64, torch.int8)
    with pytest.raises(ValueError):
        B.KvCacheStack([cache, cache])
    with pytest.raises(ValueError):
        B.KvCacheStack([cache, B.KvCache(cache.v.clone(), cache.v, cache.k_scale.clone(), cache.v_scale.clone())])


@pytest.mark.parametrize("layers,layout,page,heads,dim,dtype,fmt", SHAPES[:-1])
def test_gaps_of_many_sequences_are_closed(B, layers, layout, page, heads, dim, dtype, fmt):
    """More CTAs than SMs: whole rows, and less under way in each."""
    test_gaps_are_closed(B, layers, layout, page, heads, dim, dtype, fmt, 320, 45, 0.6)
