"""Attention to a shared prefix without suffixes (the state that merge_attn_states joins with others), and prefixes whose row blocks
and runs come out in every form, against a plain 64-bit evaluation."""
import math

import pytest
import torch

from test_gpu_shared_prefix import B, Problem  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu


def reference(p):
    """kv_reference.attend with all heads of a query token at once: (out, lse, weighted mean of |v|, largest sum of |q k| times |scale|,
    keys seen)."""
    k, v = p.kv64
    seqs, q_len, heads, dim = p.q.shape
    group = heads // p.kv_heads
    q = p.q.double().view(seqs, q_len, p.kv_heads, group, dim)
    out = torch.zeros(seqs, q_len, p.kv_heads, group, dim, dtype=torch.float64)
    lse = torch.full((seqs, q_len, p.kv_heads, group), -math.inf, dtype=torch.float64)
    mean_abs, score_abs, seen = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(lse)

    def entries(pages, n):
        at = torch.arange(n)
        page, off = pages.long()[at // p.page], at % p.page
        return k[page, off], v[page, off]

    prefix = entries(p.prefix_pages, p.prefix)
    for b, n in enumerate(p.lens):
        if n < 0:
            continue
        own = entries(p.table[b], n)
        for i in range(q_len):
            sees = max(0, n - q_len + i + 1)
            kk, vv = (torch.cat([a, c[:sees]]) for a, c in zip(prefix, own))
            if kk.shape[0] == 0:
                continue
            s = torch.einsum("hgd,khd->hgk", q[b, i], kk) * p.scale
            lse[b, i] = torch.logsumexp(s, -1)
            w = torch.exp(s - lse[b, i].unsqueeze(-1))
            out[b, i] = torch.einsum("hgk,khd->hgd", w, vv)
            mean_abs[b, i] = torch.einsum("hgk,khd->hgd", w, vv.abs())
            score_abs[b, i] = torch.einsum("hgd,khd->hgk", q[b, i].abs(), kk.abs()).amax(-1) * abs(p.scale)
            seen[b, i] = kk.shape[0]
    whole, flat = (seqs, q_len, heads, dim), (seqs, q_len, heads)
    return out.view(whole), lse.view(flat), mean_abs.view(whole), score_abs.view(flat), seen.view(flat)


ALONE = [  # seqs, prefix, heads, kv_heads, dim, page, q_len
    (40, 128, 32, 8, 128, 16, 1),    # 160 rows: one wide block and one run, hence one part
    (64, 100, 32, 8, 128, 16, 1),    # 256 rows, the only tile ends early
    (1, 1, 80, 1, 64, 16, 1),        # one key; a narrow block alone
    (65, 128, 1, 1, 64, 16, 1),      # a narrow block alone, its second stream without a tile
    (16, 700, 8, 1, 128, 24, 1),     # 128 rows: a narrow block alone, several runs
    (75, 100, 4, 1, 64, 16, 1),      # 300 rows: a wide block and a narrow one, one run
    (75, 1300, 4, 1, 96, 16, 1),     # the same with several runs
    (20, 90, 16, 1, 80, 8, 8),       # 2560 rows of one key/value head
    (1280, 200, 32, 32, 64, 16, 1),  # 160 blocks: more than there are SMs
    (5, 40, 8, 2, 128, 16, 1),       # few rows: keys first, the only part is the result
    (3, 5000, 8, 8, 64, 16, 2),      # few rows, many parts
    (40, 700, 8, 2, 256, 16, 1),     # heads of 256
]


@pytest.mark.parametrize("fmt", ["plain", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", ALONE, ids=[f"{s[0]}x{s[6]}_p{s[1]}_{s[2]}of{s[3]}x{s[4]}_page{s[5]}" for s in ALONE])
def test_prefix_without_suffixes(B, dtype, fmt, shape):
    seqs, prefix, heads, kv_heads, dim, page, q_len = shape
    lens = [-1 if i % 11 == 7 else 0 for i in range(seqs)]
    p = Problem(B, lens, prefix, heads, kv_heads, dim, page, dtype, fmt, q_len, seed=prefix + seqs)
    assert p.batch.page_table is None and p.batch.struct.max_suffix_len == 0
    ws = B.shared_prefix_attention_workspace(p.cache, p.batch, heads)
    ws.fill_(255)  # NaN: nothing of it may survive
    out, lse = p.launch(workspace=ws)
    p.check(out, lse, reference(p))
    again, lse_again = p.launch()
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse, lse_again)


@pytest.mark.parametrize("fmt", ["plain", "int8"])
@pytest.mark.parametrize("shape", [(70, 128, 1, 1, 128, 16, 1), (20, 700, 5, 1, 64, 16, 1), (16, 300, 8, 1, 96, 16, 1),  # narrow blocks alone
                                   (320, 150, 75, 75, 64, 16, 1), (150, 4000, 40, 40, 128, 16, 2)])                      # more blocks than SMs
def test_row_blocks_with_suffixes(B, fmt, shape):
    seqs, prefix, heads, kv_heads, dim, page, q_len = shape
    lens = [-1 if i % 11 == 7 else (i * 5) % 23 for i in range(seqs)]
    p = Problem(B, lens, prefix, heads, kv_heads, dim, page, "bf16", fmt, q_len, seed=prefix)
    p.check(*p.launch(), reference(p))


def test_prefix_alone_in_a_graph(B):
    p = Problem(B, [0, 0, -1, 0] * 12, 128, 32, 8, 128, 16, seed=3)
    ref = reference(p)
    q, ws = p.q.cuda(), B.shared_prefix_attention_workspace(p.cache, p.batch, p.heads)
    out, lse = torch.full_like(q, 3.0), torch.full(q.shape[:-1], 3.0, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.shared_prefix_attention_launch(p.cache, p.batch, q, out, lse, ws, softmax_scale=p.scale)
    for _ in range(2):
        out.fill_(3.0)
        lse.fill_(3.0)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        p.check(out, lse, ref)


@pytest.mark.parametrize("seqs,heads,prefix", [(40, 16, 128), (6, 16, 75), (64, 32, 900)])
def test_prefix_and_suffixes_apart_then_merged(B, oracle_lib, seqs, heads, prefix):
    """The prefix alone, the suffixes alone, and merge_attn_states: the state of the call that takes both.  Each state is within its
    own bound of the 64-bit one; the merge, of the states as they are, is held to its own oracle; and all three together to the sum of
    the bounds, the mean of the states' bounds being at most the larger."""
    import kv_reference as R
    lens = [(i * 7) % 40 for i in range(seqs)]
    whole = Problem(B, lens, prefix, heads, 4, 128, 16, seed=seqs)
    ref, ref_lse, mean_abs, score_abs, seen = reference(whole)
    q = whole.q.cuda()
    states = []
    for batch in (B.PrefixBatch(whole.prefix_pages.cuda(), prefix, None, whole.dev_lens.clamp_max(0), 0),
                  B.PrefixBatch(None, 0, whole.table.cuda(), whole.dev_lens, whole.most)):
        out, lse = torch.empty_like(q), torch.empty(q.shape[:-1], device="cuda")
        B.shared_prefix_attention_launch(whole.cache, batch, q, out, lse, softmax_scale=whole.scale)
        states.append((out[:, 0].contiguous(), lse[:, 0].contiguous()))
    (a, s_a), (b, s_b) = states
    empty = torch.tensor(lens) == 0
    assert bool((b.cpu()[empty] == 0).all()) and bool((s_b.cpu()[empty] == -math.inf).all())
    merged, s = torch.empty_like(a), torch.empty_like(s_a)
    B.SpecTable.default().launch_merge_attn_states(a, s_a, b, s_b, merged, s)
    v_ref, s_ref = oracle_lib.merge_attn_states(a.cpu(), s_a.cpu(), b.cpu(), s_b.cpu())
    assert oracle_lib.compare_mixed(merged.cpu(), v_ref, tol=2.0, tol_abs=1e-5)[1] == 0
    assert oracle_lib.compare_mixed(s.cpu(), s_ref, tol=1e-5, tol_abs=1e-5)[1] == 0
    # out = (w_a a + w_b b) / (w_a + w_b): errors of a and b are weighted, and so are the magnitudes of which the bounds are shares;
    # their own rounding to bf16 is 2^-8 of mean_abs at most, and an error e of a log-sum-exp moves the weights by e of |a|, |b|.
    lse_tol = R.lse_tolerance(ref_lse, score_abs, seen, 128)[:, 0]
    tol = R.out_tolerance(ref, mean_abs, score_abs, seen, torch.bfloat16, False, 128)[:, 0] + mean_abs[:, 0] * (2.0 ** -8 + 4 * lse_tol.unsqueeze(-1))
    assert bool(((merged.cpu().double() - ref[:, 0]).abs() <= tol).all())
    assert bool(((s.cpu().double() - ref_lse[:, 0]).abs() <= 2 * lse_tol).all())
    assert B.rt_device_status() == 0
