"""Results in the place of keys or values, which other rows still have to read, are refused, without a GPU (pointers are numbers that nothing follows)."""
import pytest

from paper_2601_12698_b200 import binding as B
from test_prompt_host import P, _call

Q, K, V, OUT, LSE = (P + (i << 20) for i in range(5))


@pytest.mark.parametrize("out", [K, V])
def test_results_over_keys_or_values_are_refused(out):
    assert _call(q=Q, k=K, v=V, out=out, lse=LSE) == B.RT_ERR_SHAPE and "overlap" in B.lib.rt_last_error().decode()
