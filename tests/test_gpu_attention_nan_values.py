"""Values that are not finite in a quantised cache (their scale is NaN): the rows that see them come out as NaN, the log-sum-exp, in
which values have no part, is that of the scores."""
import pytest
import torch

import kv_reference as R
from test_gpu_prefix_alone import reference
from test_gpu_shared_prefix import B, Problem  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu


def _check_lse(p, lse, ref):
    _, ref_lse, _, score_abs, seen = ref
    live = torch.tensor(p.lens) >= 0
    off = (lse.cpu().double() - ref_lse).abs() - R.lse_tolerance(ref_lse, score_abs, seen, p.dim)
    assert bool((off[live] <= 0).all()), f"lse beyond its bound by {off[live].max()}"


FORMS = [  # lens, prefix, heads, kv_heads, dim, q_len
    ([70, 200, -1, 33], 0, 8, 2, 128, 3),       # suffixes, 16 rows to a CTA
    ([70, 200, -1, 33], 150, 8, 2, 64, 1),      # few rows: prefix and suffixes in one launch
    ([70, 200, 33], 300, 64, 2, 256, 2),        # 64 rows to a CTA
    ([3, 9, 0, -1] * 12, 300, 8, 2, 128, 1),    # the tiles form, narrow
    ([3, 9, 0, -1] * 12, 300, 32, 2, 64, 1),    # the tiles form, wide
    ([0, -1, 0] * 30, 120, 8, 2, 128, 1),       # the tiles form, a prefix alone
]


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("lens,prefix,heads,kv_heads,dim,q_len", FORMS)
def test_a_value_scale_that_is_not_finite(B, fmt, bad, lens, prefix, heads, kv_heads, dim, q_len):
    group, seqs = heads // kv_heads, len(lens)
    p = Problem(B, lens, prefix, heads, kv_heads, dim, 16, "bf16", fmt, q_len, seed=prefix + 1)
    ref = reference(p)
    out0, lse0 = p.launch()
    p.check(out0, lse0, ref)
    # one key/value head at a time: a key of the prefix, and keys of sequence 1's suffix that only some query tokens see
    spoiled = torch.zeros(seqs, q_len, heads, dtype=torch.bool)
    if prefix:
        at = prefix - 2
        p.cache.v_scale[int(p.prefix_pages[at // 16]), at % 16, 1] = bad
        spoiled[:, :, group:2 * group] = True
    if max(lens) > 0:
        at = lens[1] - 1  # seen by the last query token only
        p.cache.v_scale[int(p.table[1, at // 16]), at % 16, 0] = bad
        spoiled[1, q_len - 1, :group] = True
    spoiled[torch.tensor(lens) < 0] = False
    assert bool(spoiled.any()) and not bool(spoiled.all())
    out, lse = p.launch()
    assert bool(torch.isnan(out.float())[spoiled].all())
    assert torch.equal(out[~spoiled], out0[~spoiled]) and torch.equal(lse[~spoiled], lse0[~spoiled])
    _check_lse(p, lse, ref)
    assert B.rt_device_status() == 0


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("seqs", [3, 40])
def test_an_infinite_value_written_into_the_cache(B, fmt, seqs):
    p = Problem(B, [5] * seqs, 200, 8, 2, 128, 16, "bf16", fmt, seed=2)
    g = torch.Generator().manual_seed(1)
    key, value = (torch.randn(1, 2, 128, generator=g).bfloat16() for _ in range(2))
    value[0, 0, 17] = float("-inf")
    slot = int(p.prefix_pages[3]) * 16 + 4
    B.kv_cache_write_launch(p.cache, key.cuda(), value.cuda(), torch.tensor([slot], device="cuda"))
    p.kv64[0].view(-1, 2, 128)[slot] = R.dequantise(*R.quantise(key[0], fmt))
    ref = reference(p)
    out, lse = p.launch()
    assert bool(torch.isnan(out[..., :4, :].float()).all()) and bool(torch.isfinite(out[..., 4:, :].float()).all())
    _check_lse(p, lse, ref)
    assert B.rt_device_status() == 0


@pytest.mark.parametrize("fmt", ["plain", "e4m3", "int8"])
@pytest.mark.parametrize("seqs", [3, 40])
def test_a_nan_value_in_a_part_that_weighs_next_to_nothing(B, fmt, seqs):
    """A key's weight is above zero however low its score: its NaN reaches the row although the part that holds it is some 2^-400 of
    the other."""
    p = Problem(B, [5] * seqs, 130, 8, 2, 64, 16, "bf16", fmt, seed=5)
    q = torch.zeros(seqs, 1, 8, 64).bfloat16()
    q[..., 0] = 300.0
    p.q, p.scale = q, 1.0
    k = p.cache.k if fmt == "plain" else p.cache.k.view(torch.uint8)
    for b in range(seqs):
        if fmt == "plain":
            k[int(p.table[b, 0]), :5, :, 0] = 1.0
        else:
            p.cache.k_scale[int(p.table[b, 0]), :5] = 1.0
            k[int(p.table[b, 0]), :5, :, 0] = 0x38 if fmt == "e4m3" else 1  # 1.0 either way
    pages = p.prefix_pages.long().cuda()
    if fmt == "plain":
        k[pages, :, :, 0] = 0.0
        p.cache.v[int(p.prefix_pages[2]), 3, 0, 9] = float("nan")
    else:
        k[pages, :, :, 0] = 0
        p.cache.v_scale[int(p.prefix_pages[2]), 3, 0] = float("nan")
    out, lse = p.launch()
    hit = out[:, 0, :4].float()
    assert bool(torch.isnan(hit[..., 9] if fmt == "plain" else hit).all())
    assert bool(torch.isfinite(out[:, 0, 4:].float()).all()) and bool(torch.isfinite(lse).all())
    assert B.rt_device_status() == 0
