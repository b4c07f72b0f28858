"""What a stack of caches accepts, without a GPU (the caches are stand-ins that nothing follows)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2601_12698_b200 import binding as B
from test_kv_cache_host import _cache


def _stand_in(n_pages, quantised=False):
    shape = (n_pages, 8, 2, 64)
    k, v = torch.zeros(shape), torch.zeros(shape)
    scales = (torch.zeros(shape[:3]), torch.zeros(shape[:3])) if quantised else (None, None)
    return SimpleNamespace(device_index=0, struct=_cache(n_pages=n_pages), k=k, v=v, k_scale=scales[0], v_scale=scales[1])


@pytest.mark.parametrize("quantised", [False, True])
def test_empty_caches_are_not_one_another(quantised):
    B.KvCacheStack([_stand_in(0, quantised)])
    B.KvCacheStack([_stand_in(0, quantised), _stand_in(0, quantised)])
    cache = _stand_in(3, quantised)
    with pytest.raises(ValueError, match="twice"):
        B.KvCacheStack([cache, cache])
