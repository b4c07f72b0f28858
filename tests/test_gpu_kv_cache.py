"""The paged key/value cache: writes and reads against the plain 64-bit form, bit for bit, and what must stay untouched."""
import pytest
import torch

import kv_reference as R

pytestmark = pytest.mark.gpu
TD = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2601_12698_b200 import binding
    torch.cuda.set_device(0)
    return binding


def _cache(B, layout, pages, page, heads, dim, dtype, fmt):
    """A cache in one of the layouts that serving programs use, every byte of it a canary."""
    held = {"plain": TD[dtype], "e4m3": torch.float8_e4m3fn, "int8": torch.int8}[fmt]
    raw = torch.uint8 if fmt != "plain" else held
    if layout == "token":
        base = [torch.full((pages, page, heads, dim), 77, dtype=raw, device="cuda") for _ in range(2)]
        k, v = base
    elif layout == "head":  # [pages, heads, page, dim]
        base = [torch.full((pages, heads, page, dim), 77, dtype=raw, device="cuda") for _ in range(2)]
        k, v = (t.permute(0, 2, 1, 3) for t in base)
    else:  # one tensor for both sides, rows with a gap
        base = [torch.full((pages, 2, page, heads, dim + 16), 77, dtype=raw, device="cuda")]
        k, v = base[0][:, 0, ..., :dim], base[0][:, 1, ..., :dim]
    scales = [None, None]
    if fmt != "plain":
        k, v = k.view(held) if k.is_contiguous() else _as(k, held), v.view(held) if v.is_contiguous() else _as(v, held)
        scales = [torch.full((pages, page, heads), 7.0, device="cuda") for _ in range(2)]
    return B.KvCache(k, v, *scales), base


def _as(t, dtype):
    return t.view(dtype)  # same element size: any strides


def _bits(t):
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def _tokens(n, heads, dim, dtype, seed, fused):
    g = torch.Generator().manual_seed(seed)
    both = torch.randn(n, 2 * heads, dim, generator=g) * torch.exp(torch.randn(n, 2 * heads, 1, generator=g) * 3)
    both = both.to(TD[dtype]).cuda()
    if fused:
        return both[:, :heads], both[:, heads:]
    return both[:, :heads].contiguous(), both[:, heads:].contiguous()


@pytest.mark.parametrize("fmt", ["plain", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n,heads,dim,page,layout,fused", [
    (1, 1, 128, 16, "token", False), (7, 2, 64, 1, "token", True), (130, 8, 128, 16, "token", True), (33, 5, 100, 24, "token", True),
    (65, 3, 33, 8, "head", False), (50, 4, 256, 64, "head", True), (21, 2, 80, 16, "gap", True), (9, 40, 128, 32, "gap", False),
    (700, 8, 128, 64, "token", False), (3, 2, 1, 4, "token", True), (12, 1, 250, 7, "head", True)])
def test_write_then_read_matches_the_definition(B, dtype, fmt, n, heads, dim, page, layout, fused):
    pages = -(-n // page) + 2
    cache, base = _cache(B, layout, pages, page, heads, dim, dtype, fmt)
    before = [t.clone() for t in base]
    key, value = _tokens(n, heads, dim, dtype, n + dim, fused)
    g = torch.Generator().manual_seed(1)
    slots = torch.randperm(pages * page, generator=g)[:n].cuda()
    if n > 5:
        slots[2] = -1
        slots[n - 1] = -7
    key[n // 2] = 0.0  # a vector of zeros
    B.kv_cache_write_launch(cache, key, value, slots)
    live = (slots >= 0).cpu()
    at = slots.cpu()[live]
    for x, held, scale in ((key, cache.k, cache.k_scale), (value, cache.v, cache.v_scale)):
        x = x.cpu()[live]
        got = held.reshape(-1, heads, dim).cpu()[at] if held.dtype != torch.float8_e4m3fn else held.view(torch.uint8).reshape(-1, heads, dim).cpu()[at]
        if fmt == "plain":
            assert torch.equal(_bits(got), _bits(x))
            continue
        codes, scales = R.quantise(x, fmt)
        got_scale = scale.reshape(-1, heads).cpu()[at]
        assert R.same(got_scale, scales)
        finite = torch.isfinite(scales)  # draws beyond fp16's range are infinities
        assert torch.equal(got.view(torch.uint8)[finite], codes.view(torch.uint8)[finite])
        # what comes back is within half a step of what went in (e4m3: 2^-4 of the value, or 2^-10 units near zero; int8: half a
        # unit), plus the binary32 roundings of scale, inverse and product, each 2^-24 of a value of at most M units
        unit = scales.double().unsqueeze(-1)
        back, x64 = codes.float().double() * unit, x.double()
        tol = x64.abs() * 2.0 ** -4 + unit * 2.0 ** -10 if fmt == "e4m3" else unit * 0.5
        assert bool(((back - x64).abs() <= tol + unit * R.CODE_MAX[fmt] * 2.0 ** -22)[finite].all())
    # nothing else was written: clear the entries written and compare with the start
    touched = torch.zeros(pages * page, dtype=torch.bool, device="cuda")
    touched[slots[slots >= 0]] = True
    for held, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        rows = held if fmt == "plain" else held.view(torch.uint8)
        assert bool((rows.reshape(-1, heads, dim)[~touched] == 77).all())
        if scale is not None:
            assert bool((scale.reshape(-1, heads)[~touched] == 7.0).all())
    if layout == "gap":
        assert torch.equal(base[0][..., dim:], before[0][..., dim:])
    # read back, out of order, one slot twice, a padded row left as it was
    order = torch.cat([slots[slots >= 0].flip(0), slots[slots >= 0][:1], torch.tensor([-1], device="cuda")])
    wide = torch.full((order.shape[0], heads, dim + 8), 5.0, dtype=TD[dtype], device="cuda")
    k_out = wide[..., :dim]
    v_out = torch.full((order.shape[0], heads, dim), 5.0, dtype=TD[dtype], device="cuda")
    B.kv_cache_read_launch(cache, order, k_out, v_out)
    assert bool((wide[..., dim:] == 5.0).all())
    for out, held, scale in ((k_out, cache.k, cache.k_scale), (v_out, cache.v, cache.v_scale)):
        assert bool((out[-1] == 5.0).all())
        rows = (held if fmt == "plain" else held.view(torch.uint8)).reshape(-1, heads, dim)[order[:-1]].cpu()
        if fmt == "plain":
            assert torch.equal(_bits(out[:-1].cpu()), _bits(rows))
        else:
            unit = scale.reshape(-1, heads)[order[:-1]].cpu()
            want = R.dequantise(rows.view(R.CODE_TYPE[fmt]), unit).float().to(TD[dtype])  # one binary32 product, rounded once
            assert R.same(out[:-1].cpu(), want)
    assert B.rt_device_status() == 0


@pytest.mark.parametrize("fmt", ["plain", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim", [4, 8, 12, 16, 20, 24, 40, 48, 60, 68, 72, 112, 124, 132, 136, 144, 248, 252])
def test_vectors_that_end_inside_a_lanes_share(B, dtype, fmt, dim):
    test_write_then_read_matches_the_definition(B, dtype, fmt, 37, 3, dim, 5, "gap" if dim % 16 else "token", dim % 3 == 0)


@pytest.mark.parametrize("fmt", ["plain", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("off", [1, 2, 4, 8])
def test_slices_that_start_off_the_vector_alignment(B, dtype, fmt, off):
    n, heads, dim, page = 45, 3, 64, 8
    g = torch.Generator().manual_seed(off)
    base = torch.randn(n, 2 * heads, dim + 16, generator=g).to(TD[dtype]).cuda()
    key, value = base[:, :heads, off:off + dim], base[:, heads:, off:off + dim]
    cache, _ = _cache(B, "token", 8, page, heads, dim, dtype, fmt)
    slots = torch.randperm(8 * page, generator=g)[:n].cuda()
    B.kv_cache_write_launch(cache, key, value, slots)
    wide = [torch.full((n, heads, dim + 16), 5.0, dtype=TD[dtype], device="cuda") for _ in range(2)]
    out = [t[..., off:off + dim] for t in wide]
    B.kv_cache_read_launch(cache, slots, *out)
    for x, y, t in ((key, out[0], wide[0]), (value, out[1], wide[1])):
        if fmt == "plain":
            want = x.cpu()
        else:
            codes, scales = R.quantise(x.cpu(), fmt)
            want = R.dequantise(codes, scales).float().to(TD[dtype])
        assert torch.equal(y.cpu(), want)
        assert bool((t[..., :off] == 5.0).all()) and bool((t[..., off + dim:] == 5.0).all())
    assert B.rt_device_status() == 0


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_values_that_are_hard_to_quantise(B, dtype, fmt):
    """Infinities and NaN make the whole vector NaN and only it; the largest and smallest finite values and exact ties round as defined."""
    dim, big = 64, torch.finfo(TD[dtype]).max
    rows = torch.ones(10, 1, dim)
    rows[0, 0, 3] = float("inf")
    rows[1, 0, 5] = float("-inf")
    rows[2, 0, 7] = float("nan")
    rows[3] = big
    rows[4] = torch.linspace(-1, 1, dim) * min(big, 1e30)
    rows[5] = 0.0
    rows[6] = torch.finfo(TD[dtype]).smallest_normal / 4
    rows[7] = torch.arange(dim).float() - 31.5  # halves: ties of the int8 rounding once scaled by 127 / 31.5
    rows[8] = torch.pow(2.0, -torch.arange(dim).float() / 4)
    rows[9] = 1e-13
    rows = rows.to(TD[dtype]).cuda()
    cache = B.KvCache.allocate(3, 4, 1, dim, R.CODE_TYPE[fmt])
    slots = torch.arange(10, device="cuda")
    B.kv_cache_write_launch(cache, rows, rows.clone(), slots)
    back_k, back_v = torch.empty_like(rows), torch.empty_like(rows)
    B.kv_cache_read_launch(cache, slots, back_k, back_v)
    assert torch.equal(_bits(back_k[3:]), _bits(back_v[3:]))
    assert bool(torch.isnan(back_k[:3].float()).all()) and bool(torch.isnan(back_v[:3].float()).all())
    codes, scales = R.quantise(rows[3:].cpu(), fmt)
    assert torch.equal(cache.k_scale.reshape(-1)[3:10].cpu(), scales.reshape(-1))
    assert torch.equal(cache.k.view(torch.uint8).reshape(-1, dim)[3:10].cpu(), codes.view(torch.uint8).reshape(-1, dim))


def test_slots_beyond_the_cache_are_skipped_and_reported(B):
    cache = B.KvCache.allocate(4, 8, 2, 64, torch.int8)
    x = torch.randn(5, 2, 64, device="cuda", dtype=torch.bfloat16)
    slots = torch.tensor([0, 32, 5, 1 << 40, 31], device="cuda")
    assert B.rt_device_status() == 0
    B.kv_cache_write_launch(cache, x, x, slots)
    assert B.rt_device_status() == B.RT_ERR_INDEX and B.rt_device_status() == 0
    written = (cache.k_scale.reshape(-1, 2) != 0).all(-1).nonzero().flatten().tolist()
    assert written == [0, 5, 31]
    out = [torch.full_like(x, 9.0) for _ in range(2)]
    B.kv_cache_read_launch(cache, slots, *out)
    assert B.rt_device_status() == B.RT_ERR_INDEX
    for o in out:
        assert bool((o[[1, 3]] == 9.0).all()) and not bool((o[[0, 2, 4]] == 9.0).any())


def test_offsets_past_32_bits(B):
    """Pages of a cache of 4.5 GB a side, at its very end."""
    page, heads, dim = 64, 8, 128
    pages = (9 << 29) // (page * heads * dim)
    k, v = (torch.empty(pages, page, heads, dim, dtype=torch.int8, device="cuda") for _ in range(2))
    scales = [torch.zeros(pages, page, heads, device="cuda") for _ in range(2)]
    cache = B.KvCache(k, v, *scales)
    x = torch.randn(6, 2, heads, dim, device="cuda").bfloat16()
    slots = torch.tensor([0, page, pages * page - 1, pages * page - page, (pages // 2) * page, (1 << 32) // (heads * dim)], device="cuda")
    B.kv_cache_write_launch(cache, x[:, 0], x[:, 1], slots)
    out = [torch.empty(6, heads, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.kv_cache_read_launch(cache, slots, *out)
    for side in range(2):
        codes, unit = R.quantise(x[:, side].cpu(), "int8")
        assert torch.equal(_bits(out[side].cpu()), _bits(R.dequantise(codes, unit).float().bfloat16()))
    assert B.rt_device_status() == 0


def test_empty_call_other_stream_and_graph(B):
    cache = B.KvCache.allocate(4, 16, 2, 64, torch.float8_e4m3fn)
    none = torch.empty(0, 2, 64, device="cuda", dtype=torch.bfloat16)
    before = B.rt_launch_count()
    B.kv_cache_write_launch(cache, none, none, torch.empty(0, dtype=torch.int64, device="cuda"))
    B.kv_cache_read_launch(cache, torch.empty(0, dtype=torch.int64, device="cuda"), none, none)
    assert B.rt_launch_count() == before
    x = torch.randn(20, 2, 64, device="cuda").half()
    slots = torch.arange(20, device="cuda") + 11
    k_out, v_out = torch.zeros_like(x), torch.zeros_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.kv_cache_write_launch(cache, x, x, slots)
        B.kv_cache_read_launch(cache, slots, k_out, v_out)
    for seed in range(3):  # new inputs in the captured tensors
        x.copy_(torch.randn(20, 2, 64, generator=torch.Generator().manual_seed(seed)).half())
        slots.copy_(torch.randperm(64, generator=torch.Generator().manual_seed(seed))[:20])
        graph.replay()
        torch.cuda.synchronize()
        codes, unit = R.quantise(x.cpu(), "e4m3")
        want = R.dequantise(codes, unit).float().half()
        assert torch.equal(_bits(k_out.cpu()), _bits(want)) and torch.equal(_bits(v_out.cpu()), _bits(want))
    B.kv_cache_read_launch(cache, slots, k_out.zero_(), v_out, stream=None)
    torch.cuda.synchronize()
    k_out.zero_()
    torch.cuda.synchronize()
    B.kv_cache_read_launch(cache, slots, k_out, v_out, stream=side)
    side.synchronize()
    assert torch.equal(_bits(k_out.cpu()), _bits(want))


def test_binding_refuses_what_does_not_fit(B):
    cache = B.KvCache.allocate(4, 16, 2, 64, torch.int8)
    x = torch.zeros(3, 2, 64, device="cuda", dtype=torch.bfloat16)
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    for key, value, s in ((x.cpu(), x, slots), (x, x[:2], slots), (x, x.half(), slots), (x, x, slots.int()), (x.transpose(1, 2), x, slots),
                          (x, x, slots.cpu()), (x[:, :1], x[:, :1], slots)):
        with pytest.raises(ValueError):
            B.kv_cache_write_launch(cache, key, value, s)
    with pytest.raises(ValueError):
        B.kv_cache_read_launch(cache, slots, x[:1].expand(3, 2, 64), x)
    plain = B.KvCache.allocate(4, 16, 2, 64, torch.float16)
    with pytest.raises(B.TunerError) as e:
        B.kv_cache_write_launch(plain, x, x, slots)
    assert e.value.status == B.RT_ERR_DTYPE
    k = torch.zeros(4, 16, 2, 64, dtype=torch.int8, device="cuda")
    scale = torch.zeros(4, 16, 2, device="cuda")
    for args in ((k, k), (k, k, scale, None), (k, k[:2], scale, scale), (k.bfloat16(), k.bfloat16(), scale, scale), (k, k, scale.half(), scale.half()),
                 (k.cpu(), k.cpu(), scale, scale), (k[:, :, :, :1].expand(4, 16, 2, 64), k[:, :, :, :1].expand(4, 16, 2, 64), scale, scale)):
        with pytest.raises(ValueError):
            B.KvCache(*args)
