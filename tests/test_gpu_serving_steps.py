"""Rotary positions, the cache, attention over packed prompts and over the cache, forked pages and given-up drafts in one run, as a serving
program uses them, against a plain 64-bit form that keeps every sequence's keys in a list of its own."""

import pytest
import torch

import kv_reference as R
import prompt_reference as P
from test_gpu_prompt import B  # noqa: F401  (a fixture)
from test_gpu_rotary import reference as turned

pytestmark = pytest.mark.gpu
HEADS, KV, DIM, PAGE, LAYERS = 8, 2, 64, 16, 3


class Layer:
    """What one layer's projections give for some tokens, and the keys and values of every sequence so far (CPU, bf16)."""

    def __init__(self, seed):
        self.g = torch.Generator().manual_seed(seed)
        self.held = {}

    def project(self, n):
        return (torch.randn(n, HEADS + 2 * KV, DIM, generator=self.g) * 1.5).to(torch.bfloat16)


def _attend(q, keys, values, first):
    """One sequence's queries (bf16) from position `first` on, and what the tolerance wants."""
    n = q.shape[0]
    out, lse, mean_abs, score_abs, seen, _ = P.attend(q, keys[:first + n], values[:first + n], [0, n], [0, first + n], True, DIM ** -0.5)
    return out, lse, mean_abs, score_abs, seen


def _check(got_out, got_lse, refs):
    out, lse, mean_abs, score_abs, seen = (torch.cat(x) for x in zip(*refs))
    tol = R.out_tolerance(out, mean_abs, score_abs, seen, torch.bfloat16, False, DIM)
    assert not bool(((got_out.double().cpu().reshape(out.shape) - out).abs() > tol).any())
    assert not bool(((got_lse.double().cpu().reshape(lse.shape) - lse).abs() > R.lse_tolerance(lse, score_abs, seen, DIM)).any())


def test_prompt_chunk_fork_draft_and_compact(B):
    table = B.RotaryTable(DIM // 2, base=50000.0, scaling="yarn", factor=4.0, original_len=512, interleaved=True)
    n_pages, width = 64, 12
    caches = [B.KvCache.allocate(n_pages, PAGE, KV, DIM, torch.bfloat16) for _ in range(LAYERS)]
    stack = B.KvCacheStack(caches)
    layers = [Layer(i) for i in range(LAYERS)]
    free = torch.randperm(n_pages, generator=torch.Generator().manual_seed(9)).tolist()
    pages, lens = {}, {}

    def grow(seq, n):
        lens[seq] = lens.get(seq, 0) + n
        mine = pages.setdefault(seq, [])
        while len(mine) * PAGE < lens[seq]:
            mine.append(free.pop())

    def slots(seq, first, n):
        return [pages[seq][p // PAGE] * PAGE + p % PAGE for p in range(first, first + n)]

    def table_of(seqs):
        t = torch.zeros(len(seqs), width, dtype=torch.int32)
        for i, s in enumerate(seqs):
            t[i, :len(pages[s])] = torch.tensor(pages[s], dtype=torch.int32)
        return t.cuda()

    def run_layer(layer, cache, seqs, counts, starts):
        """Projects, turns and writes `counts` tokens of `seqs` from positions `starts` on; returns the turned queries and, on the device, q, k, v."""
        fused = layer.project(sum(counts)).cuda()
        q, k, v = fused[:, :HEADS], fused[:, HEADS:HEADS + KV], fused[:, HEADS + KV:]
        positions = torch.tensor([p for s, n, a in zip(seqs, counts, starts) for p in range(a, a + n)])
        want, bound = turned(table, positions.tolist(), torch.cat([q, k], 1).cpu(), False)
        B.rotary_launch(table, positions.cuda(), q, k)
        got = torch.cat([q, k], 1).cpu()
        step = torch.finfo(torch.bfloat16).eps / 2
        assert not bool(((got.double() - want).abs() > bound * (1 + step) + step * want.abs()).any())
        B.kv_cache_write_launch(cache, k, v, torch.tensor([x for s, n, a in zip(seqs, counts, starts) for x in slots(s, a, n)]).cuda())
        at = 0
        for s, n in zip(seqs, counts):
            old = layer.held.get(s, (torch.zeros(0, KV, DIM, dtype=torch.bfloat16),) * 2)
            layer.held[s] = tuple(torch.cat([o, x[at:at + n].cpu()]) for o, x in zip(old, (k, v)))
            at += n
        return q, k, v

    # 1. three prompts, packed
    seqs, counts = [0, 1, 2], [70, 1, 33]
    for s, n in zip(seqs, counts):
        grow(s, n)
    starts_d = torch.tensor([0, 70, 71, 104], dtype=torch.int32, device="cuda")
    batch = B.PromptBatch(starts_d, 70)
    for layer, cache in zip(layers, caches):
        q, k, v = run_layer(layer, cache, seqs, counts, [0, 0, 0])
        out, lse = torch.empty(104, HEADS, DIM, dtype=torch.bfloat16, device="cuda"), torch.empty(104, HEADS, device="cuda")
        B.prompt_attention_launch(batch, q, k, v, out, lse)
        at, refs = 0, []
        for s, n in zip(seqs, counts):
            refs.append(_attend(q[at:at + n].cpu(), *layer.held[s], 0))
            at += n
        _check(out, lse, refs)

    # 2. a chunk more of two of them, behind what the cache holds
    more, counts, firsts = [0, 2], [20, 40], [70, 33]
    for s, n in zip(more, counts):
        grow(s, n)
    q_starts, k_starts = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 20, 60], [0, 90, 163]))
    batch = B.PromptBatch(q_starts, 40, k_starts, 90)
    for layer, cache in zip(layers, caches):
        q, _, _ = run_layer(layer, cache, more, counts, firsts)
        k, v = (torch.empty(163, KV, DIM, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        B.kv_cache_read_launch(cache, torch.tensor(slots(0, 0, 90) + slots(2, 0, 73)).cuda(), k, v)
        out, lse = torch.empty(60, HEADS, DIM, dtype=torch.bfloat16, device="cuda"), torch.empty(60, HEADS, device="cuda")
        B.prompt_attention_launch(batch, q, k, v, out, lse)
        _check(out, lse, [_attend(q[:20].cpu(), *layer.held[0], 70), _attend(q[20:].cpu(), *layer.held[2], 33)])

    # 3. a fork of sequence 0: whole pages shared, its last, partly filled one copied in all layers
    pages[3], lens[3] = pages[0][:-1] + [free.pop()], lens[0]
    B.kv_cache_copy_pages_launch(stack, torch.tensor([pages[0][-1]], dtype=torch.int32, device="cuda"), torch.tensor([pages[3][-1]], dtype=torch.int32, device="cuda"),
                                 torch.tensor([lens[0] % PAGE], dtype=torch.int32, device="cuda"))
    for layer in layers:
        layer.held[3] = layer.held[0]

    # 4. five drafted tokens each, attended to over the cache; then the accepted ones close up
    seqs, before = [0, 1, 2, 3], [lens[s] for s in (0, 1, 2, 3)]
    for s in seqs:
        grow(s, 5)

    def decode(n_new, firsts):
        for layer, cache in zip(layers, caches):
            q, _, _ = run_layer(layer, cache, seqs, [n_new] * 4, firsts)
            step = B.PrefixBatch(None, 0, table_of(seqs), torch.tensor([lens[s] for s in seqs], dtype=torch.int32, device="cuda"), max(lens.values()), q_len=n_new)
            q = q.contiguous().view(4, n_new, HEADS, DIM)
            out, lse = torch.empty_like(q), torch.empty(4, n_new, HEADS, device="cuda")
            B.shared_prefix_attention_launch(cache, step, q, out, lse)
            refs = [_attend(q[i].cpu(), *layer.held[s], a) for i, (s, a) in enumerate(zip(seqs, firsts))]
            _check(out, lse, refs)

    decode(5, before)
    keep = torch.tensor([[1, 1, 0, 0, 0], [1, 0, 1, 0, 1], [0, 0, 0, 0, 0], [1, 1, 1, 1, 1]], dtype=torch.bool)
    new = torch.empty(4, dtype=torch.int32, device="cuda")
    B.kv_cache_compact_launch(stack, table_of(seqs), torch.tensor(before, dtype=torch.int32, device="cuda"),
                              torch.tensor([lens[s] for s in seqs], dtype=torch.int32, device="cuda"), keep.cuda(), new)
    assert new.tolist() == [a + int(k.sum()) for a, k in zip(before, keep)]
    for i, s in enumerate(seqs):
        lens[s] = int(new[i])
        kept = torch.cat([torch.ones(before[i], dtype=torch.bool), keep[i]])
        for layer in layers:
            layer.held[s] = tuple(x[kept] for x in layer.held[s])

    # 5. one token more of everything, on the closed-up cache
    firsts = [lens[s] for s in seqs]
    for s in seqs:
        grow(s, 1)
    decode(1, firsts)
    assert B.rt_device_status() == 0
