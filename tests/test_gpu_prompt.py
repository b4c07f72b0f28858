"""Attention over packed prompts against the plain 64-bit form, element by element; tolerances as derived in kv_reference.py."""
import math

import pytest
import torch

import kv_reference as R
import prompt_reference as P

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
    """One batch: lens = [(queries, keys)] of the sequences; `tail` rows behind the last one; fused: k and v are slices of one tensor."""

    def __init__(self, B, lens, heads, kv_heads, dim, dtype="bf16", causal=True, tail=0, seed=0, spread=1.0, fused=True):
        g = torch.Generator().manual_seed(seed)
        self.B, self.dtype, self.causal, self.dim = B, TD[dtype], causal, dim
        self.q_starts, self.k_starts = [0], [0]
        for a, b in lens:
            self.q_starts.append(self.q_starts[-1] + a)
            self.k_starts.append(self.k_starts[-1] + b)
        rows, keys = self.q_starts[-1] + tail, self.k_starts[-1] + tail
        self.q = (torch.randn(rows, heads, dim, generator=g) * spread).to(self.dtype).cuda()
        both = torch.randn(keys, 2 * kv_heads, dim, generator=g)
        both[:, kv_heads:] *= torch.exp(0.5 * torch.randn(2 * kv_heads, dim, generator=g))[kv_heads:]
        both = both.to(self.dtype).cuda()
        self.k, self.v = both[:, :kv_heads], both[:, kv_heads:]
        if not fused:
            self.k, self.v = self.k.contiguous(), self.v.contiguous()
        self.scale = dim ** -0.5
        self.lens = lens
        self.batch = self.make_batch(max(a for a, _ in lens), max(b for _, b in lens))

    def starts(self):
        return [torch.tensor(s, dtype=torch.int32, device="cuda") for s in (self.q_starts, self.k_starts)]

    def make_batch(self, max_q, max_k):
        q, k = self.starts()
        return self.B.PromptBatch(q, max_q, k, max_k, causal=self.causal)

    def launch(self, batch=None, workspace=None, stream=None):
        out = torch.full(self.q.shape, 5.0, dtype=self.dtype, device="cuda")
        lse = torch.full(self.q.shape[:2], 5.0, device="cuda")
        self.B.prompt_attention_launch(batch or self.batch, self.q, self.k, self.v, out, lse, workspace, softmax_scale=self.scale, stream=stream)
        return out, lse

    def reference(self):
        return P.attend(self.q.cpu(), self.k.cpu(), self.v.cpu(), self.q_starts, self.k_starts, self.causal, self.scale)

    def check(self, out, lse, ref=None):
        want, want_lse, mean_abs, score_abs, seen, live = ref or self.reference()
        out, lse = out.double().cpu(), lse.double().cpu()
        assert torch.equal(out[~live], torch.full_like(out[~live], 5.0)) and torch.equal(lse[~live], torch.full_like(lse[~live], 5.0))
        none = seen == 0
        empty = none & live[:, None]
        assert bool((out[empty] == 0).all()) and bool((lse[empty] == -math.inf).all())
        some = ~none
        tol = R.out_tolerance(want, mean_abs, score_abs, seen, self.dtype, False, self.dim)
        bad = (out - want).abs() > tol
        assert not bool(bad[some].any()), (int(bad[some].sum()), float((out - want).abs()[some].max()))
        lse_bad = (lse - want_lse).abs() > R.lse_tolerance(want_lse, score_abs, seen, self.dim)
        assert not bool(lse_bad[some].any())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("lens,heads,kv_heads,dim", [
    ([(1, 1)], 1, 1, 128), ([(128, 128)], 1, 1, 128), ([(100, 100)], 8, 2, 128), ([(300, 300)], 4, 1, 64), ([(257, 257)], 2, 2, 256), ([(129, 129)], 5, 1, 128),
    ([(64, 64), (0, 0), (1, 1), (200, 200), (33, 33)], 4, 2, 128), ([(7, 7)] * 20, 8, 1, 80), ([(5, 5), (300, 300)], 6, 2, 96), ([(70, 70), (20, 20)], 2, 1, 8),
    ([(40, 40), (3, 3)], 3, 1, 136), ([(90, 90), (128, 128), (256, 256)], 16, 2, 64), ([(50, 50)], 128, 1, 64), ([(9, 9), (30, 30)], 65, 1, 128), ([(700, 700)], 2, 1, 128),
    ([(1, 1)] * 200, 4, 4, 64), ([(31, 31), (290, 290)], 8, 8, 256), ([(60, 60)], 7, 7, 40)])
def test_causal_prompts(B, dtype, lens, heads, kv_heads, dim):
    p = Problem(B, lens, heads, kv_heads, dim, dtype, tail=3, seed=len(lens) + dim)
    p.check(*p.launch())
    assert B.rt_device_status() == 0


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,heads,kv_heads,dim", [
    ([(1, 1000)], 8, 2, 128), ([(16, 900), (1, 1), (5, 130)], 4, 1, 128), ([(100, 1500)], 5, 1, 64), ([(3, 700), (0, 40), (64, 64)], 4, 4, 256),
    ([(1, n) for n in (0, 1, 127, 128, 129, 256, 1000)], 8, 2, 128), ([(200, 80), (10, 0), (4, 3), (300, 150)], 4, 2, 128), ([(2, 5000)], 2, 1, 96), ([(130, 2000)] * 3, 2, 2, 256)])
def test_more_or_fewer_keys_than_queries(B, causal, lens, heads, kv_heads, dim):
    p = Problem(B, lens, heads, kv_heads, dim, "bf16", causal, tail=2, seed=len(lens))
    p.check(*p.launch())
    assert B.rt_device_status() == 0


def test_the_length_hints_change_roundings_alone(B):
    p = Problem(B, [(40, 3000), (5, 2000), (0, 100)], 8, 2, 128, seed=4)
    ref = p.reference()
    sizes = set()
    for max_q, max_k in ((40, 3000), (1, 1), (0, 0), (1 << 20, 1 << 20), (40, 1024), (1, 1 << 20)):
        batch = p.make_batch(max_q, max_k)
        sizes.add(B.prompt_attention_workspace_bytes(batch, p.q, p.k))
        p.check(*p.launch(batch), ref)
    assert len(sizes) > 1  # with parts and without


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("spread", [0.0, 4.0, 20.0])
def test_scores_far_apart_and_all_alike(B, dim, spread):
    """The reference of a row moves often, or never."""
    p = Problem(B, [(300, 600), (64, 64)], 4, 1, dim, "fp16", seed=7, spread=spread)
    ref = p.reference()
    p.check(*p.launch(), ref)
    # scores that ascend along the keys: every tile moves the reference
    p.k.copy_((p.k.float() * torch.linspace(0.1, 3.0, p.k.shape[0], device="cuda")[:, None, None]).to(p.dtype))
    p.check(*p.launch())


def test_a_scale_of_zero_is_the_mean(B):
    p = Problem(B, [(70, 70), (5, 300)], 4, 2, 128, seed=3)
    p.scale = 0.0
    p.check(*p.launch())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim,heads,kv_heads", [(128, 4, 2), (64, 5, 1), (256, 2, 1), (136, 2, 2)])
@pytest.mark.parametrize("parts", [False, True])
def test_infinities_and_nan_reach_only_the_rows_that_see_them(B, dtype, dim, heads, kv_heads, parts):
    p = Problem(B, [(150, 1300 if parts else 150), (3, 3), (40, 40)], heads, kv_heads, dim, dtype, tail=130, seed=dim)
    n0 = p.lens[0][1]
    p.v[n0 - 30, 0, 3] = math.inf          # seen by the last 30 rows of the first sequence
    p.v[n0 - 10, 0, 5] = math.nan
    p.v[n0 - 5, 0, dim - 1] = -math.inf
    p.v[n0 - 3, 0, dim - 1] = math.inf     # both infinities of one column: NaN from here on
    p.k[n0 - 20, kv_heads - 1, 0] = math.nan
    p.v[n0 + 3 + 39, :, 1] = math.inf      # the last row of the last sequence
    p.k[p.k_starts[-1]:] = math.nan        # rows of no sequence
    p.v[p.k_starts[-1]:] = math.inf
    out, lse = (t.double().cpu() for t in p.launch())
    want, want_lse, mean_abs, score_abs, seen, live = p.reference()
    live[:] &= True
    assert torch.equal(torch.isnan(out[live]), torch.isnan(want[live]))
    inf = torch.isinf(want) & live[:, None, None]
    assert torch.equal(out[inf], want[inf]) and torch.equal(torch.isinf(out[live]), torch.isinf(want[live]))
    assert torch.equal(torch.isnan(lse[live]), torch.isnan(want_lse[live]))
    fine = torch.isfinite(want) & live[:, None, None]
    tol = R.out_tolerance(want, mean_abs, torch.nan_to_num(score_abs, nan=0.0), seen, p.dtype, False, dim)
    assert not bool(((out - want).abs() > tol)[fine].any())


def test_huge_values_of_hidden_keys_do_not_count(B):
    for dtype, huge in (("bf16", 3e38), ("fp16", 65504.0)):
        p = Problem(B, [(100, 100), (40, 30)], 4, 2, 128, dtype, tail=100, seed=8)
        want = p.launch()
        p.v[50:100] = huge
        p.v[100 + 20:] = -huge
        out, lse = p.launch()
        rows = list(range(50)) + list(range(100, 130))  # they see none of those keys
        assert torch.equal(out[rows], want[0][rows]) and torch.equal(lse, want[1])


def test_nan_queries_stay_in_their_rows(B):
    p = Problem(B, [(200, 200), (50, 50)], 4, 2, 128, seed=2)
    clean_out, clean_lse = p.launch()
    p.q[17, 1] = math.nan
    p.q[230, 3, 5] = math.inf
    out, lse = p.launch()
    bad = torch.zeros(250, 4, dtype=torch.bool, device="cuda")
    bad[17, 1] = bad[230, 3] = True
    assert bool(torch.isnan(out[bad]).all()) and bool(torch.isnan(lse[17, 1]))
    assert torch.equal(out[~bad], clean_out[~bad]) and torch.equal(lse[~bad], clean_lse[~bad])


def test_strides_layouts_and_slices(B):
    lens = [(90, 90), (200, 200)]
    p = Problem(B, lens, 4, 2, 64, seed=9, fused=False)
    want = p.launch()
    q, k, v = p.q, p.k, p.v
    p.q = q.permute(1, 0, 2).contiguous().permute(1, 0, 2)                    # heads outermost
    p.k = k.permute(1, 0, 2).contiguous().permute(1, 0, 2)
    for a, b in zip(p.launch(), want):
        assert torch.equal(a, b)
    wide = torch.zeros(290, 3, 4, 80, dtype=q.dtype, device="cuda")            # gaps everywhere
    wide[:, 1, :, 8:72] = q
    p.q, p.k = wide[:, 1, :, 8:72], k
    for a, b in zip(p.launch(), want):
        assert torch.equal(a, b)
    p.v = torch.cat([v, v], 0)[:290]                                           # another allocation
    for a, b in zip(p.launch(), want):
        assert torch.equal(a, b)


def test_results_repeat_bit_for_bit_and_without_lse(B):
    p = Problem(B, [(600, 600), (3, 2500)], 8, 2, 128, seed=1)
    out, lse = p.launch()
    for _ in range(3):
        again, lse2 = p.launch()
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    alone = torch.full_like(out, 5.0)
    B.prompt_attention_launch(p.batch, p.q, p.k, p.v, alone, softmax_scale=p.scale)
    assert torch.equal(alone, out)
    B.prompt_attention_launch(p.batch, p.q, p.k, p.v, alone)  # the default scale
    assert torch.equal(alone, out)


def test_many_sequences_and_many_blocks(B):
    """More sequences than a warp keeps in registers, more items than CTAs; the blocks' order is by cost."""
    g = torch.Generator().manual_seed(0)
    lens = [(int(n), int(n) + int(c)) for n, c in zip(torch.randint(0, 40, (300,), generator=g), torch.randint(0, 3, (300,), generator=g) * 50)]
    lens[150] = (900, 900)
    for causal in (True, False):
        p = Problem(B, lens, 2, 2, 64, "bf16", causal, tail=1, seed=5)
        p.check(*p.launch())


@pytest.mark.parametrize("keys", [70, 3000])
def test_starts_that_descend_or_lie_outside_are_reported_and_nothing_is_written(B, keys):
    """With parts (many keys) and without."""
    p = Problem(B, [(50, 50), (60, 60), (70, keys)], 2, 1, 64, seed=1)
    q, k = p.starts()
    end = 110 + keys
    B.rt_device_status()
    for bad_q, bad_k in (([0, 50, 110, 5000], None), ([0, 50, 40, 180], None), ([-5, 50, 110, 180], None), (None, [0, 50, 110, 1 << 30]), (None, [0, 120, 110, end]),
                         ([0, 180, 0, 180], None), ([0, 50, 110, -1], None)):
        qs = q if bad_q is None else torch.tensor(bad_q, dtype=torch.int32, device="cuda")
        ks = k if bad_k is None else torch.tensor(bad_k, dtype=torch.int32, device="cuda")
        out, lse = torch.full_like(p.q, 5.0), torch.full(p.q.shape[:2], 5.0, device="cuda")
        B.prompt_attention_launch(B.PromptBatch(qs, 70, ks, keys), p.q, p.k, p.v, out, lse)
        assert B.rt_device_status() == B.RT_ERR_INDEX
        assert bool((out == 5.0).all()) and bool((lse == 5.0).all())
    p.check(*p.launch())
    assert B.rt_device_status() == 0


def test_bad_starts_among_many_sequences(B):
    """The one that is wrong is looked up, not kept in a register."""
    p = Problem(B, [(3, 3)] * 400, 2, 2, 64, seed=1)
    q, _ = p.starts()
    for at in (5, 200, 399):
        bad = q.clone()
        bad[at] = 1 << 20
        out = torch.full_like(p.q, 5.0)
        B.prompt_attention_launch(B.PromptBatch(bad, 3), p.q, p.k, p.v, out)
        assert B.rt_device_status() == B.RT_ERR_INDEX and bool((out == 5.0).all())


def test_streams_graphs_and_workspaces(B):
    p = Problem(B, [(30, 4000), (2, 3000)], 8, 2, 128, seed=6)
    size = B.prompt_attention_workspace_bytes(p.batch, p.q, p.k)
    assert size > 0
    ref = p.reference()
    want = p.launch()
    p.check(*want, ref)
    spaces = [B.prompt_attention_workspace(p.batch, p.q, p.k) for _ in range(2)]
    sides = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [p.launch(workspace=w, stream=s) for w, s in zip(spaces, sides)] + [p.launch(stream=sides[0])]
    torch.cuda.synchronize()
    for out, lse in got:
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    out, lse = torch.full_like(want[0], 5.0), torch.full_like(want[1], 5.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.prompt_attention_launch(p.batch, p.q, p.k, p.v, out, lse, spaces[0], softmax_scale=p.scale)
    spaces[0].fill_(255)  # it carries nothing from call to call
    p.v.mul_(2)
    graph.replay()
    p.check(out, lse)
    p.check(*p.launch())


def test_an_expired_wait_is_reported_and_the_next_call_is_right(B):
    from test_gpu_timeout import _expiring_waits
    for lens, heads, kv_heads, dim in (([(300, 300), (20, 20)], 4, 1, 128), ([(40, 2000)], 2, 1, 64), ([(200, 200)] * 3, 2, 2, 256)):
        p = Problem(B, lens, heads, kv_heads, dim, seed=1)
        ref = p.reference()
        p.check(*p.launch(), ref)
        with _expiring_waits(B, polls=50):
            p.launch()
            assert B.rt_device_status() == B.RT_ERR_DEVICE_TIMEOUT
            assert B.rt_device_status() == 0
        for _ in range(2):
            p.check(*p.launch(), ref)


def test_refusals(B):
    p = Problem(B, [(30, 30)], 4, 2, 64, seed=1)
    out = torch.empty_like(p.q)
    good = dict(q=p.q, k=p.k, v=p.v, out=out)
    for bad in (dict(q=p.q[0]), dict(q=p.q.float()), dict(k=p.k.half()), dict(v=p.v[:20]), dict(k=p.k[..., :32]), dict(out=out[:20]), dict(out=out.transpose(0, 1)), dict(q=p.q.cpu()),
                dict(q=p.q.transpose(1, 2)), dict(lse=torch.empty(30, 4)), dict(lse=torch.empty(30, 4, dtype=torch.float64, device="cuda"))):
        with pytest.raises(ValueError):
            B.prompt_attention_launch(p.batch, **{**good, **bad})
    for bad in (dict(q=p.q[:, :3].contiguous(), out=out[:, :3].contiguous()), dict(softmax_scale=-1.0), dict(k=p.k[:1].expand(30, 2, 64), v=p.v)):
        with pytest.raises((ValueError, B.TunerError)):
            B.prompt_attention_launch(p.batch, **{**good, **bad})
    q, k = p.starts()
    for bad in (dict(q_starts=q.long()), dict(q_starts=q.cpu()), dict(k_starts=k[:1]), dict(max_q_len=-1), dict(max_k_len=-1)):
        with pytest.raises(ValueError):
            B.PromptBatch(**{**dict(q_starts=q, max_q_len=30, k_starts=k, max_k_len=30), **bad})
    long = Problem(B, [(4, 4000)], 4, 1, 64, seed=1)
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.TunerError) as e:
        long.launch(workspace=small)
    assert e.value.status == B.RT_ERR_CAPACITY


@pytest.mark.parametrize("dim,causal", [(256, True), (200, True), (256, False), (128, True)])
def test_many_short_blocks_to_a_cta(B, dim, causal):
    """One block's results leave while the next one's products are under way, eleven blocks to a CTA and more."""
    lens = [(1 + 7 * i % 40, 1 + 7 * i % 40 + (61 * i % 190 if i % 3 else 0)) for i in range(420)]
    p = Problem(B, lens, 4, 4, dim, seed=3, causal=causal)
    first = p.launch()
    p.check(*first)
    for _ in range(4):
        assert all(torch.equal(a, b) for a, b in zip(first, p.launch()))
    assert B.rt_device_status() == 0


@pytest.mark.parametrize("n", [127, 128, 129, 161, 700])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 256])
def test_many_sequences_of_very_different_costs(B, n, causal, dim):
    """Every block is taken once, whatever the order: costs from nothing to many blocks of keys, empty sequences among them."""
    g = torch.Generator().manual_seed(n)
    q = (torch.rand(n, generator=g) ** 12 * 900).int().tolist()
    more = (torch.rand(n, generator=g) ** 6 * 1200).int().tolist()
    p = Problem(B, [(a, a + b if i % 5 else b) for i, (a, b) in enumerate(zip(q, more))], 4, 2, dim, tail=3, seed=n, causal=causal)
    p.check(*p.launch())
    assert B.rt_device_status() == 0
