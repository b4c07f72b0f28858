"""As many sequences as the attention over packed prompts takes, nearly all of them empty."""
import pytest
import torch

import kv_reference as R
import prompt_reference as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2601_12698_b200 import binding
    torch.cuda.set_device(0)
    return binding


def test_blocks_of_many_costs_among_many_sequences(B):
    """Single queries behind keys of ten powers of two.  Who takes the cheapest block goes through all sequences ten times, some seconds'
    tenths each: longer than the second that a wait for a copy is given."""
    n, dim = 1 << 24, 64
    g = torch.Generator().manual_seed(1)
    lens = [(1, 5), *[(1, 256 << i) for i in range(9)]]
    at = sorted(torch.randperm(n, generator=g)[:len(lens)].tolist())
    q_lens, k_lens = torch.zeros(n, dtype=torch.int32), torch.zeros(n, dtype=torch.int32)
    for i, (a, b) in zip(at, lens):
        q_lens[i], k_lens[i] = a, b
    q_starts, k_starts = (torch.cat([torch.zeros(1, dtype=torch.int32), torch.cumsum(x, 0).int()]).cuda() for x in (q_lens, k_lens))
    rows, keys = sum(a for a, _ in lens), sum(b for _, b in lens)
    q, k, v = (torch.randn(m, 1, dim, generator=g).bfloat16().cuda() for m in (rows, keys, keys))
    out, lse = torch.empty_like(q), torch.empty(rows, 1, device="cuda")
    B.rt_device_status()
    batch = B.PromptBatch(q_starts, 1, k_starts, max(b for _, b in lens))
    B.prompt_attention_launch(batch, q, k, v, out, lse, softmax_scale=0.125)
    assert B.rt_device_status() == 0
    dense = [[0, *torch.tensor(x).cumsum(0).tolist()] for x in zip(*lens)]
    want, want_lse, mean_abs, score_abs, seen, _ = P.attend(q.cpu(), k.cpu(), v.cpu(), *dense, True, 0.125)
    assert not bool(((out.cpu().double() - want).abs() > R.out_tolerance(want, mean_abs, score_abs, seen, q.dtype, False, dim)).any())
    assert not bool(((lse.cpu().double() - want_lse).abs() > R.lse_tolerance(want_lse, score_abs, seen, dim)).any())
