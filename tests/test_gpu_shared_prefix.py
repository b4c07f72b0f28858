"""Attention over a shared prefix and a paged cache against a plain 64-bit evaluation."""
import math

import pytest
import torch

import kv_reference as R

pytestmark = pytest.mark.gpu
TD = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2601_12698_b200 import binding
    torch.cuda.set_device(0)
    return binding


class Problem:
    """A batch, its cache (CPU in 64 bits and on the device) and its queries.  Every entry of the cache that no sequence owns is
    NaN, scales included; so are the page numbers that no sequence needs (out of range)."""

    def __init__(self, B, lens, prefix, heads, kv_heads, dim, page, dtype="bf16", fmt="plain", q_len=1, layout="token", seed=0, spread=1.0,
                 most=None, scale=None):
        g = torch.Generator().manual_seed(seed)
        self.B, self.lens, self.prefix, self.dtype, self.fmt, self.q_len, self.page = B, list(lens), prefix, dtype, fmt, q_len, page
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        seqs = len(self.lens)
        self.most = max([0, *self.lens]) if most is None else most
        width = max(1, -(-self.most // page))
        need = [-(-max(0, n) // page) for n in self.lens]
        n_prefix = -(-prefix // page)
        pages = n_prefix + sum(need) + 3
        order = torch.randperm(pages, generator=g).to(torch.int32)
        self.prefix_pages = order[:n_prefix].clone()
        table = torch.full((seqs, width), 1 << 20, dtype=torch.int32)
        at = n_prefix
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.table = table
        kv = torch.randn(2, pages, page, kv_heads, dim, generator=g) * torch.exp(0.5 * torch.randn(2, 1, 1, kv_heads, dim, generator=g)) * spread
        owned = torch.zeros(pages, page, dtype=torch.bool)
        for i in range(prefix):
            owned[int(self.prefix_pages[i // page]), i % page] = True
        for b, n in enumerate(self.lens):
            for i in range(max(0, n)):
                owned[int(table[b, i // page]), i % page] = True
        self.owned = owned
        held, scales, self.kv64 = [], [None, None], []
        for side in range(2):
            x = kv[side].to(TD[dtype])
            if fmt == "plain":
                x[~owned] = float("nan")
                held.append(x)
                self.kv64.append(x.double())
            else:
                codes, unit = R.quantise(x, fmt)
                unit[~owned] = float("nan")
                if fmt == "e4m3":
                    codes.view(torch.uint8)[~owned] = 0x7F
                held.append(codes)
                scales[side] = unit
                self.kv64.append(R.dequantise(codes, unit))
        held = [self._lay_out(t, layout) for t in held]
        self.cache = B.KvCache(*held, *[None if t is None else t.cuda() for t in scales])
        self.q = torch.randn(seqs, q_len, heads, dim, generator=g).to(TD[dtype])
        self.scale = dim ** -0.5 if scale is None else scale
        self.dev_lens = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.batch = self.make_batch()

    def make_batch(self):
        return self.B.PrefixBatch(self.prefix_pages.cuda() if self.prefix else None, self.prefix, self.table.cuda() if self.most else None,
                                  self.dev_lens, self.most, self.q_len)

    @staticmethod
    def _lay_out(t, layout):
        raw = t.view(torch.uint8) if t.element_size() == 1 else t
        if layout == "token":
            d = raw.cuda()
        elif layout == "head":
            d = raw.cuda().permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
        else:  # rows with a gap, sides of one tensor
            pages, page, heads, dim = raw.shape
            d = torch.full((pages, 2, page, heads, dim + 32), 1, dtype=raw.dtype, device="cuda")[:, 1, ..., :dim]
            d.copy_(raw)
        return d.view(t.dtype) if t.element_size() == 1 else d

    def launch(self, q=None, **kw):
        q = self.q.cuda() if q is None else q
        out = torch.full(self.q.shape, 3.0, dtype=self.q.dtype, device="cuda")
        lse = torch.full(self.q.shape[:-1], 3.0, dtype=torch.float32, device="cuda")
        self.B.shared_prefix_attention_launch(self.cache, self.batch, q, out, lse, softmax_scale=self.scale, **kw)
        return out, lse

    def reference(self):
        k, v = self.kv64
        return R.attend(k, v, self.prefix_pages, self.prefix, self.table, self.lens, self.q, self.scale)

    def check(self, out, lse, reference=None):
        ref, ref_lse, mean_abs, score_abs, seen = reference or self.reference()
        out, lse = out.cpu().double(), lse.cpu().double()
        dead = torch.tensor(self.lens) < 0
        assert bool((out[dead] == 3.0).all()) and bool((lse[dead] == 3.0).all()), "a padded sequence's rows were written"
        out, lse, ref, ref_lse = out[~dead], lse[~dead], ref[~dead], ref_lse[~dead]
        mean_abs, score_abs, seen = mean_abs[~dead], score_abs[~dead], seen[~dead]
        tol = R.out_tolerance(ref, mean_abs, score_abs, seen, TD[self.dtype], self.fmt != "plain", self.dim)
        empty = seen == 0
        assert bool((out[empty] == 0).all()) and bool((lse[empty] == -math.inf).all())
        off = (out - ref).abs() - tol
        assert bool((off[~empty] <= 0).all()), f"out beyond its bound by {off[~empty].max()}, at most {tol.max()} allowed"
        off = ((lse - ref_lse).abs() - R.lse_tolerance(ref_lse, score_abs, seen, self.dim))[~empty]
        assert bool((off <= 0).all()), f"lse beyond its bound by {off.max()}"
        assert self.B.rt_device_status() == 0


SHAPES = [  # lens, prefix, heads, kv_heads, dim, page, q_len
    ([1], 0, 1, 1, 64, 16, 1),
    ([1, 0, 5], 1, 4, 4, 128, 16, 1),
    ([0, 0], 77, 8, 2, 128, 16, 1),
    ([200, 3, -1, 64, 65, 0], 130, 8, 2, 128, 16, 1),
    ([33, 15, 16, 17, 31], 1000, 32, 8, 128, 64, 1),
    ([5, 300], 0, 10, 2, 64, 1, 1),
    ([40, 2, 0, 130], 65, 12, 4, 96, 24, 3),
    ([3, 1, 9], 0, 16, 1, 80, 8, 5),
    ([90, -1, 16, 2], 257, 16, 1, 256, 32, 2),
    ([600, 599, 1], 300, 5, 5, 64, 128, 16),
    ([7, 12], 20, 40, 8, 128, 7, 1),
    ([1, 2, 3, 4, 5, 6, 7, 8, 9, 10] * 7, 129, 16, 2, 64, 16, 1),
    ([75], 300, 16, 1, 64, 16, 3),
    ([300], 400, 24, 1, 256, 16, 2),
]


@pytest.mark.parametrize("fmt", ["plain", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES, ids=[f"{len(s[0])}x{s[6]}_p{s[1]}_{s[2]}of{s[3]}x{s[4]}_page{s[5]}" for s in SHAPES])
def test_matches_the_plain_form(B, dtype, fmt, shape):
    lens, prefix, heads, kv_heads, dim, page, q_len = shape
    p = Problem(B, lens, prefix, heads, kv_heads, dim, page, dtype, fmt, q_len, seed=len(lens) + prefix)
    out, lse = p.launch()
    p.check(out, lse)
    again, lse_again = p.launch()
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse, lse_again)


@pytest.mark.parametrize("layout", ["head", "gap"])
@pytest.mark.parametrize("fmt", ["plain", "e4m3", "int8"])
def test_layouts_and_strided_queries(B, fmt, layout):
    p = Problem(B, [30, 9, 70], 90, 8, 2, 128, 16, "bf16", fmt, 2, layout=layout, seed=5)
    fused = torch.full((6, 8 + 4, 128), float("nan"), dtype=torch.bfloat16, device="cuda")  # a fused projection: q, then k and v
    fused[:, :8] = p.q.cuda().view(6, 8, 128)
    q = fused.view(3, 2, 12, 128)[:, :, :8]
    p.check(*p.launch(q=q))


@pytest.mark.parametrize("fmt", ["plain", "e4m3", "int8"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 20.0])
def test_scales_of_the_scores(B, fmt, scale):
    """No preference, an inverted one, and scores of hundreds, where one key takes all."""
    p = Problem(B, [50, 3, 128], 100, 8, 2, 64, 16, "bf16", fmt, seed=9, scale=scale)
    p.check(*p.launch())


@pytest.mark.parametrize("fmt,spread", [("plain", 1e-20), ("plain", 1e4), ("e4m3", 1e-9), ("e4m3", 3e4), ("int8", 3e4), ("int8", 1e-9)])
def test_magnitudes_of_keys_and_values(B, fmt, spread):
    """Values far from 1, whose scales would leave fp16's range if the weights carried them."""
    p = Problem(B, [50, 3, 128], 100, 8, 2, 64, 16, "bf16", fmt, seed=10, spread=spread, scale=0.1 / spread if spread > 1 else 0.1)
    p.check(*p.launch())


@pytest.mark.parametrize("dtype,fmt", [("bf16", "plain"), ("fp16", "plain"), ("bf16", "e4m3")])
def test_hidden_keys_have_no_influence(B, dtype, fmt):
    """A drafted token's infinite or NaN key and value reach the query tokens that see it and no other."""
    lens, q_len = [40, 20], 4
    p = Problem(B, lens, 50, 8, 2, 128, 16, dtype, fmt, q_len, seed=3)
    clean = p.reference()
    out0, lse0 = p.launch()
    page, off = int(p.table[0, 38 // 16]), 38 % 16  # key 38: seen by query tokens 2 and 3 of sequence 0
    if fmt == "plain":
        p.cache.v[page, off, 0, 3] = float("inf")
        p.cache.v[page, off, 0, 77] = float("-inf")
        p.cache.v[page, off, 1, 5] = float("nan")
        p.cache.k[int(p.table[0, 39 // 16]), 39 % 16, :, 9] = float("nan")  # key 39: seen by token 3 only
    else:
        p.cache.v.view(torch.uint8)[page, off, 0, 3] = 0x7F
        p.cache.v.view(torch.uint8)[page, off, 1, 5] = 0xFF
        p.cache.v_scale[int(p.table[0, 39 // 16]), 39 % 16, :] = float("nan")
    out, lse = p.launch()
    torch.cuda.synchronize()
    assert torch.equal(out[1], out0[1]) and torch.equal(lse[1], lse0[1])
    assert torch.equal(out[0, :2], out0[0, :2]) and torch.equal(lse[0, :2], lse0[0, :2])
    row = out[0, 2].float()
    head0 = row[:4]  # query heads of key/value head 0
    if fmt == "plain":
        assert bool((head0[:, 3] == math.inf).all()) and bool((head0[:, 77] == -math.inf).all()) and bool(torch.isnan(row[4:, 5]).all())
        hit = torch.zeros_like(row, dtype=torch.bool)
        hit[:4, 3] = hit[:4, 77] = hit[4:, 5] = True
    else:
        assert bool(torch.isnan(head0[:, 3]).all()) and bool(torch.isnan(row[4:, 5]).all())
        hit = torch.zeros_like(row, dtype=torch.bool)
        hit[:4, 3] = hit[4:, 5] = True
    assert torch.equal(row[~hit], out0[0, 2].float()[~hit])
    assert bool(torch.isnan(out[0, 3].float()).all())
    assert B.rt_device_status() == 0
    del clean


def test_visible_infinities_and_nan(B):
    """What a row does see reaches it: an infinite value gives an infinite output in its column, a NaN key a NaN row."""
    p = Problem(B, [20, 20], 40, 4, 1, 64, 16, seed=4)
    p.cache.v[int(p.prefix_pages[1]), 2, 0, 11] = float("inf")
    p.cache.k[int(p.table[1, 0]), 3, 0, 0] = float("nan")
    out, lse = p.launch()
    assert bool((out[0, 0, :, 11].float() == math.inf).all()) and bool(torch.isfinite(out[0, 0, :, :11].float()).all())
    assert bool(torch.isnan(out[1].float()).all()) and bool(torch.isnan(lse[1]).all()) and bool(torch.isfinite(lse[0]).all())


def test_pages_outside_the_cache_are_hidden_and_reported(B):
    p = Problem(B, [40, 20], 48, 4, 2, 64, 16, seed=6)
    p.table[0, 1] = 10 ** 6
    p.prefix_pages[2] = -3
    p.batch = p.make_batch()
    assert B.rt_device_status() == 0
    out, lse = p.launch()
    assert B.rt_device_status() == B.RT_ERR_INDEX and B.rt_device_status() == 0
    # the same batch without those keys
    k, v = p.kv64
    prefix_pages, table = p.prefix_pages[:2], torch.stack([p.table[0, [0, 2, 2]], p.table[1]])
    ref = R.attend(k, v, prefix_pages, 32, table, [24, 20], p.q, p.scale)
    p.check(out, lse, ref)


def test_lengths_beyond_the_declared_one_are_cut_and_reported(B):
    p = Problem(B, [40, 20], 48, 4, 2, 64, 16, seed=7)
    p.dev_lens[0] = 1000
    out, lse = p.launch()
    assert B.rt_device_status() == B.RT_ERR_INDEX
    p.check(out, lse)


def test_padded_batch_streams_and_graphs(B):
    """One captured graph serves steps of other lengths, pages and queries; two graphs with a workspace each replay on two streams."""
    probs = [Problem(B, [30, 2, 55, -1, 7], 100, 8, 2, 128, 16, "bf16", "plain", seed=20 + i, most=64) for i in range(2)]
    graphs, bufs, streams = [], [], [torch.cuda.Stream() for _ in probs]
    for p, s in zip(probs, streams):
        q, out = p.q.cuda(), torch.full(p.q.shape, 3.0, dtype=p.q.dtype, device="cuda")
        lse = torch.full(p.q.shape[:-1], 3.0, device="cuda")
        ws = B.shared_prefix_attention_workspace(p.cache, p.batch, p.heads)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            B.shared_prefix_attention_launch(p.cache, p.batch, q, out, lse, ws, softmax_scale=p.scale)
        graphs.append(g)
        bufs.append((q, out, lse))
    for step in range(3):
        for p, (q, out, lse) in zip(probs, bufs):
            gen = torch.Generator().manual_seed(100 + step)
            p.q = torch.randn(p.q.shape, generator=gen).to(p.q.dtype)
            p.lens = [30 - step, step, 55 - 20 * step, -1 if step < 2 else 0, 7]
            q.copy_(p.q)
            out.fill_(3.0)
            lse.fill_(3.0)
            p.dev_lens.copy_(torch.tensor(p.lens, dtype=torch.int32))
        torch.cuda.synchronize()
        for _ in range(4):
            for g, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        for p, (q, out, lse) in zip(probs, bufs):
            p.check(out, lse)


def test_options_and_outputs_that_may_be_left_out(B):
    p = Problem(B, [30, 9], 300, 8, 2, 64, 16, seed=8)
    out, lse = p.launch()
    q = p.q.cuda()
    alone = torch.empty_like(q)
    B.shared_prefix_attention_launch(p.cache, p.batch, q, alone)  # no lse, default scale, own workspace
    assert torch.equal(alone, out)
    three = torch.empty(2, 8, 64, dtype=q.dtype, device="cuda")
    B.shared_prefix_attention_launch(p.cache, p.batch, q[:, 0], three)
    assert torch.equal(three, out[:, 0])
    try:
        assert B.lib.rt_set_option(B.RT_OPTION_PROGRAMMATIC_LAUNCH, 0) == B.RT_OK
        serial, lse_serial = p.launch()
    finally:
        assert B.lib.rt_set_option(B.RT_OPTION_PROGRAMMATIC_LAUNCH, 1) == B.RT_OK
    assert torch.equal(serial, out) and torch.equal(lse_serial, lse)
    none = B.PrefixBatch(None, 0, None, torch.zeros(2, dtype=torch.int32, device="cuda"), 0)
    out, lse = torch.ones_like(three), torch.zeros(2, 8, device="cuda")
    B.shared_prefix_attention_launch(p.cache, none, q[:, 0], out, lse)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    empty = B.PrefixBatch(None, 0, None, torch.zeros(0, dtype=torch.int32, device="cuda"), 0)
    B.shared_prefix_attention_launch(p.cache, empty, q[:0, 0], out[:0])
    assert B.rt_device_status() == 0


def test_refusals(B):
    p = Problem(B, [30, 9], 20, 8, 2, 64, 16, seed=8)
    q = p.q.cuda()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:-1], device="cuda")
    launch = B.shared_prefix_attention_launch
    for args in ((q[:1], out[:1]), (q, out.float()), (q, out.transpose(1, 2)), (q, out.cpu()), (q.cpu(), out), (q[..., :32], out[..., :32]),
                 (q, out, lse.half()), (q, out, lse[:1]), (q, out, lse, torch.empty(8, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            launch(p.cache, p.batch, *args)
    before = B.rt_launch_count()
    for args, status in (((q.float(), out.float()), B.RT_ERR_DTYPE), ((q.half(), out.half()), B.RT_ERR_DTYPE),
                         ((q, out, lse, torch.empty(64, dtype=torch.uint8, device="cuda")), B.RT_ERR_CAPACITY),
                         ((q[:, :, :7].contiguous(), out[:, :, :7].contiguous()), B.RT_ERR_SHAPE)):
        with pytest.raises((B.TunerError, ValueError)) as e:
            launch(p.cache, p.batch, *args)
        if isinstance(e.value, B.TunerError):
            assert e.value.status == status
    odd = torch.empty(2 * 8 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(2, 1, 8, 64)
    with pytest.raises(B.TunerError) as e:
        launch(p.cache, p.batch, odd, out)
    assert e.value.status == B.RT_ERR_ALIGN
    with pytest.raises(B.TunerError) as e:  # no pages at all
        launch(B.KvCache.allocate(0, 16, 2, 64, torch.bfloat16), p.batch, q, out, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    assert e.value.status == B.RT_ERR_SHAPE
    assert B.rt_launch_count() == before
    for kw in ({"prefix_pages": p.prefix_pages.cuda().long()}, {"page_table": p.table.cuda()[:1]}, {"suffix_lens": p.dev_lens.long()},
               {"suffix_lens": p.dev_lens.cpu()}):
        d = {"prefix_pages": p.prefix_pages.cuda(), "page_table": p.table.cuda(), "suffix_lens": p.dev_lens, **kw}
        with pytest.raises(ValueError):
            B.PrefixBatch(d["prefix_pages"], 20, d["page_table"], d["suffix_lens"], 30)


def test_offsets_past_32_bits(B):
    """Keys whose places in the cache lie past 2^32 bytes and past 2^31 elements."""
    page, heads, dim = 64, 8, 128
    pages = (5 << 30) // (2 * page * heads * dim)
    k, v = (torch.empty(pages, page, heads, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    small = Problem(B, [70, 100], 130, 16, 8, dim, page, seed=11)
    n = small.cache.n_pages
    far = torch.arange(pages - n, pages)
    k[pages - n:], v[pages - n:] = small.cache.k, small.cache.v
    small.cache = B.KvCache(k, v)
    near_lists = small.prefix_pages.clone(), small.table.clone()
    small.prefix_pages, small.table = (torch.where(t < n, far[t.clamp_max(n - 1).long()].int(), t) for t in near_lists)
    small.batch = small.make_batch()
    out, lse = small.launch()
    small.prefix_pages, small.table = near_lists
    small.check(out, lse)


def test_cache_then_attention_then_merge(B, oracle_lib):
    """A decoding step as a server runs it: the new tokens' keys and values are written into a quantised cache, every sequence
    attends to the shared prefix and its own suffix, and the result is merged with that of a further block of keys."""
    from paper_2601_12698_b200.binding import SpecTable
    g = torch.Generator().manual_seed(2)
    seqs, heads, kv_heads, dim, page, prefix = 6, 16, 4, 128, 16, 75
    lens = [1, 20, 33, 16, 17, 2]
    cache = B.KvCache.allocate(32, page, kv_heads, dim, torch.float8_e4m3fn)
    prefix_pages = torch.arange(20, 25, dtype=torch.int32)
    table = torch.arange(18, dtype=torch.int32).view(6, 3)
    kv64 = [torch.zeros(32, page, kv_heads, dim, dtype=torch.float64) for _ in range(2)]

    def write(slots):
        x = torch.randn(len(slots), 2, kv_heads, dim, generator=g).bfloat16()
        d = x.cuda()
        B.kv_cache_write_launch(cache, d[:, 0], d[:, 1], torch.tensor(slots, device="cuda"))
        for side in range(2):
            kv64[side].view(-1, kv_heads, dim)[slots] = R.dequantise(*R.quantise(x[:, side], "e4m3"))

    write([int(prefix_pages[i // page]) * page + i % page for i in range(prefix)])
    write([int(table[b, i // page]) * page + i % page for b in range(seqs) for i in range(lens[b] - 1)])
    write([int(table[b, (lens[b] - 1) // page]) * page + (lens[b] - 1) % page for b in range(seqs)])  # this step's tokens
    batch = B.PrefixBatch(prefix_pages.cuda(), prefix, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), 48)
    q = torch.randn(seqs, 1, heads, dim, generator=g).bfloat16()
    out, lse = torch.empty_like(q, device="cuda"), torch.empty(seqs, 1, heads, device="cuda")
    B.shared_prefix_attention_launch(cache, batch, q.cuda(), out, lse)
    ref, ref_lse, mean_abs, score_abs, seen = R.attend(*kv64, prefix_pages, prefix, table, lens, q, dim ** -0.5)
    assert bool(((out.cpu().double() - ref).abs() <= R.out_tolerance(ref, mean_abs, score_abs, seen, torch.bfloat16, True, dim)).all())
    assert bool(((lse.cpu().double() - ref_lse).abs() <= R.lse_tolerance(ref_lse, score_abs, seen, dim)).all())
    other, s_other = torch.randn(seqs, heads, dim, generator=g).bfloat16(), torch.randn(seqs, heads, generator=g) + 4
    merged, s = torch.empty(seqs, heads, dim, dtype=torch.bfloat16, device="cuda"), torch.empty(seqs, heads, device="cuda")
    SpecTable.default().launch_merge_attn_states(out[:, 0].contiguous(), lse[:, 0].contiguous(), other.cuda(), s_other.cuda(), merged, s)
    v_ref, s_ref = oracle_lib.merge_attn_states(out[:, 0].cpu().contiguous(), lse[:, 0].cpu().contiguous(), other, s_other)
    assert oracle_lib.compare_mixed(merged.cpu(), v_ref, tol=2.0, tol_abs=1e-5)[1] == 0
    assert oracle_lib.compare_mixed(s.cpu(), s_ref, tol=1e-5, tol_abs=1e-5)[1] == 0
    assert B.rt_device_status() == 0


# ---- batches large enough for the tensor-core form of the prefix -------------------------------------------------------

MANY = [  # seqs, prefix, heads, kv_heads, dim, page, q_len
    (40, 128, 1, 1, 128, 16, 1),        # one tile: the second stream has none
    (40, 500, 8, 8, 64, 16, 1),         # 40 rows: narrow blocks
    (33, 1000, 8, 2, 128, 24, 1),       # 132 rows: the second stream has 4
    (70, 700, 4, 1, 96, 16, 2),         # 560 rows: two wide blocks and a narrow one
    (300, 5121, 8, 8, 64, 64, 1),       # more tiles than SMs: runs that end one unit and begin the next
    (64, 1537, 16, 4, 128, 1, 1),
    (9, 3000, 40, 8, 80, 16, 5),        # 225 rows, prefix ends inside a tile and a page
    (20, 130, 64, 1, 128, 128, 1),      # 1280 rows of one key/value head
    (40, 700, 8, 2, 256, 16, 1),        # heads of 256: 64 rows at a time, keys first
    (11, 500, 16, 2, 240, 24, 2),
    (4, 600, 64, 2, 128, 16, 2),        # 64 rows to a suffix
]


@pytest.mark.parametrize("fmt", ["plain", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", MANY, ids=[f"{s[0]}x{s[6]}_p{s[1]}_{s[2]}of{s[3]}x{s[4]}_page{s[5]}" for s in MANY])
def test_many_rows_match_the_plain_form(B, dtype, fmt, shape):
    seqs, prefix, heads, kv_heads, dim, page, q_len = shape
    lens = [-1 if i % 11 == 7 else (i * 5) % 23 for i in range(seqs)]
    p = Problem(B, lens, prefix, heads, kv_heads, dim, page, dtype, fmt, q_len, seed=prefix)
    out, lse = p.launch()
    assert B.rt_device_status() == 0
    p.check(out, lse)
    again, lse_again = p.launch()
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse, lse_again)


@pytest.mark.parametrize("fmt", ["plain", "e4m3", "int8"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 20.0])
def test_many_rows_scales_of_the_scores(B, fmt, scale):
    p = Problem(B, [3] * 40, 700, 4, 1, 64, 16, "bf16", fmt, seed=9, scale=scale)
    p.check(*p.launch())


@pytest.mark.parametrize("fmt,spread", [("plain", 1e-20), ("plain", 1e4), ("e4m3", 1e-9), ("e4m3", 3e4), ("int8", 3e4), ("int8", 1e-9)])
def test_many_rows_magnitudes(B, fmt, spread):
    p = Problem(B, [3] * 40, 700, 4, 1, 64, 16, "bf16", fmt, seed=10, spread=spread, scale=0.1 / spread if spread > 1 else 0.1)
    p.check(*p.launch())


@pytest.mark.parametrize("fmt", ["plain", "e4m3"])
def test_rising_scores_move_the_reference(B, fmt):
    """Keys whose scores rise through the prefix by far more than the margin at which a row's reference is moved."""
    p = Problem(B, [2] * 70, 1500, 4, 1, 64, 16, "bf16", fmt, seed=12)
    q = torch.ones(70, 1, 4, 64).bfloat16()
    q[::2] = -1.0
    p.q = q
    ramp = torch.linspace(-30, 30, 1500)
    for i in range(1500):
        at = int(p.prefix_pages[i // 16]), i % 16
        x = torch.full((1, 64), float(ramp[i])).bfloat16()
        if fmt == "plain":
            p.cache.k[at] = x.cuda()
            p.kv64[0][at] = x.double()
        else:
            codes, unit = R.quantise(x, fmt)
            p.cache.k.view(torch.uint8)[at] = codes.view(torch.uint8).cuda()
            p.cache.k_scale[at] = unit.cuda()
            p.kv64[0][at] = R.dequantise(codes, unit)
    p.check(*p.launch())


def test_many_rows_pages_outside_the_cache(B):
    p = Problem(B, [5] * 40, 16 * 20, 4, 1, 128, 16, seed=6)
    bad = [3, 4, 19]
    p.prefix_pages[bad] = torch.tensor([-1, 10 ** 6, p.cache.n_pages], dtype=torch.int32)
    p.batch = p.make_batch()
    assert B.rt_device_status() == 0
    out, lse = p.launch()
    assert B.rt_device_status() == B.RT_ERR_INDEX
    kept = [i for i in range(20) if i not in bad]
    k, v = p.kv64
    p.check(out, lse, R.attend(k, v, p.prefix_pages[kept], 16 * 17, p.table, p.lens, p.q, p.scale))
    p.prefix_pages[:] = -1  # nothing of the prefix is there
    p.batch = p.make_batch()
    out, lse = p.launch()
    assert B.rt_device_status() == B.RT_ERR_INDEX
    p.check(out, lse, R.attend(k, v, p.prefix_pages, 0, p.table, p.lens, p.q, p.scale))


def test_many_rows_visible_infinities_and_nan(B):
    p = Problem(B, [5] * 40, 400, 4, 1, 64, 16, seed=4)
    out0, lse0 = p.launch()
    p.cache.v[int(p.prefix_pages[20]), 2, 0, 11] = float("inf")
    out, lse = p.launch()
    assert bool((out[..., 11].float() == math.inf).all()) and torch.equal(lse, lse0)
    rest = torch.ones(64, dtype=torch.bool)
    rest[11] = False
    assert torch.equal(out[..., rest], out0[..., rest])
    q = p.q.cuda()
    q[7, 0, 1, 5] = float("nan")
    out, lse = p.launch(q=q)
    assert bool(torch.isnan(out[7, 0, 1].float()).all()) and bool(torch.isnan(lse[7, 0, 1]))
    assert int(torch.isnan(lse).sum()) == 1


def test_many_rows_in_a_graph_with_the_options(B):
    p = Problem(B, [3, 0, 9, -1] * 20, 900, 8, 2, 128, 16, seed=30)
    out, lse = p.launch()
    p.check(out, lse)
    q, ws = p.q.cuda(), B.shared_prefix_attention_workspace(p.cache, p.batch, p.heads)
    got, got_lse = torch.full_like(out, 3.0), torch.full_like(lse, 3.0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for _ in range(3):
            B.shared_prefix_attention_launch(p.cache, p.batch, q, got, got_lse, ws, softmax_scale=p.scale)
    for _ in range(2):
        ws.fill_(255)  # NaN: nothing of it may survive
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(got_lse, lse)
    try:
        assert B.lib.rt_set_option(B.RT_OPTION_PROGRAMMATIC_LAUNCH, 0) == B.RT_OK
        serial, lse_serial = p.launch()
    finally:
        assert B.lib.rt_set_option(B.RT_OPTION_PROGRAMMATIC_LAUNCH, 1) == B.RT_OK
    assert torch.equal(serial, out) and torch.equal(lse_serial, lse)


@pytest.mark.parametrize("shapes", [((40, 500, 8, 8, 64, 16, 1), (64, 1537, 16, 4, 128, 1, 1)), ((33, 1000, 8, 2, 128, 24, 1), (3, 200, 8, 2, 128, 16, 2)),
                                    ((40, 700, 8, 2, 256, 16, 1), (33, 1000, 8, 2, 128, 24, 1))])
def test_calls_behind_one_another_and_side_by_side(B, shapes):
    """Calls on one stream take turns with one workspace; calls on two streams have one each.  The results are those of a call alone."""
    problems = [Problem(B, [(7 * i) % 40 for i in range(s[0])], s[1], *s[2:6], "bf16", "plain" if n else "e4m3", s[6], seed=n) for n, s in enumerate(shapes)]
    alone = []
    for p in problems:
        alone.append(p.launch())
        torch.cuda.synchronize()
    size = max(B.shared_prefix_attention_workspace_bytes(p.cache, p.batch, p.q.shape[-2]) for p in problems)
    q = [p.q.cuda() for p in problems]
    shared = torch.empty(size, dtype=torch.uint8, device="cuda")
    behind = [[(torch.full_like(x, 3.0), torch.full(x.shape[:-1], 3.0, device="cuda")) for x in q] for _ in range(6)]
    for outs in behind:
        for p, x, (out, lse) in zip(problems, q, outs):
            B.shared_prefix_attention_launch(p.cache, p.batch, x, out, lse, workspace=shared, softmax_scale=p.scale)
    torch.cuda.synchronize()
    streams, own = [torch.cuda.Stream() for _ in problems], [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in problems]
    beside = [[(torch.full_like(x, 3.0), torch.full(x.shape[:-1], 3.0, device="cuda")) for x in q] for _ in range(6)]
    torch.cuda.synchronize()
    for outs in beside:
        for p, x, (out, lse), s, w in zip(problems, q, outs, streams, own):
            B.shared_prefix_attention_launch(p.cache, p.batch, x, out, lse, workspace=w, softmax_scale=p.scale, stream=s)
    torch.cuda.synchronize()
    for outs in behind + beside:
        for (out, lse), (want, want_lse) in zip(outs, alone):
            assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and torch.equal(lse, want_lse)
    assert B.rt_device_status() == 0
