"""Refusals of the attention over packed prompts and its struct, without a GPU (pointers are numbers that nothing follows)."""
import ctypes
import math
import os
import subprocess
import tempfile

import pytest

from paper_2601_12698_b200 import binding as B

P = 1 << 20


def _batch(**kw):
    d = dict(q_starts=P, k_starts=P, n_seqs=3, q_tokens=100, k_tokens=100, max_q_len=50, max_k_len=50, causal=1, reserved=0)
    d.update(kw)
    return B.rt_prompt_batch(**d)


def _call(batch=None, q=P, qts=512, qhs=128, heads=4, k=P, kts=256, khs=128, v=P, vts=256, vhs=128, kv_heads=2, dim=128, out=P, lse=P, scale=0.1,
          dtype=0, workspace=P, size=1 << 40):
    b = _batch() if batch is None else batch
    return B.lib.prompt_attention_launch(ctypes.byref(b), q, qts, qhs, heads, k, kts, khs, v, vts, vhs, kv_heads, dim, out, lse, scale, dtype, workspace, size, None)


GEOMETRY = [
    (dict(batch=_batch(n_seqs=-1)), "RT_ERR_SHAPE"), (dict(batch=_batch(n_seqs=(1 << 24) + 1)), "RT_ERR_SHAPE"), (dict(batch=_batch(q_tokens=-1)), "RT_ERR_SHAPE"),
    (dict(batch=_batch(q_tokens=(1 << 30) + 1)), "RT_ERR_SHAPE"), (dict(batch=_batch(k_tokens=(1 << 30) + 1)), "RT_ERR_SHAPE"),
    (dict(batch=_batch(max_q_len=-1)), "RT_ERR_SHAPE"), (dict(batch=_batch(max_k_len=-1)), "RT_ERR_SHAPE"), (dict(heads=3), "RT_ERR_SHAPE"),
    (dict(heads=0), "RT_ERR_SHAPE"), (dict(kv_heads=0), "RT_ERR_SHAPE"), (dict(heads=258, kv_heads=2), "RT_ERR_SHAPE"), (dict(dim=4), "RT_ERR_SHAPE"),
    (dict(dim=100), "RT_ERR_SHAPE"), (dict(dim=264), "RT_ERR_SHAPE")]


@pytest.mark.parametrize("kw,status", GEOMETRY + [
    (dict(dtype=2), "RT_ERR_DTYPE"), (dict(dtype=-1), "RT_ERR_DTYPE"), (dict(scale=-0.1), "RT_ERR_SHAPE"), (dict(scale=math.nan), "RT_ERR_SHAPE"),
    (dict(scale=math.inf), "RT_ERR_SHAPE"), (dict(q=None), "RT_ERR_NULL"), (dict(k=None), "RT_ERR_NULL"), (dict(v=None), "RT_ERR_NULL"), (dict(out=None), "RT_ERR_NULL"),
    (dict(batch=_batch(q_starts=None)), "RT_ERR_NULL"), (dict(batch=_batch(k_starts=None)), "RT_ERR_NULL"), (dict(q=P + 8), "RT_ERR_ALIGN"),
    (dict(v=P + 8), "RT_ERR_ALIGN"), (dict(out=P + 2), "RT_ERR_ALIGN"), (dict(lse=P + 2), "RT_ERR_ALIGN"), (dict(workspace=P + 8), "RT_ERR_ALIGN"), (dict(qts=516), "RT_ERR_ALIGN"),
    (dict(khs=132), "RT_ERR_ALIGN"), (dict(vts=0), "RT_ERR_SHAPE"), (dict(qhs=-128), "RT_ERR_SHAPE"), (dict(kts=1 << 39), "RT_ERR_SHAPE"),
    (dict(batch=_batch(q_starts=P + 2)), "RT_ERR_ALIGN")])
def test_launch_refusals(kw, status):
    assert _call(**kw) == getattr(B, status)
    assert B.lib.rt_last_error()


@pytest.mark.parametrize("kw,status", GEOMETRY)
def test_workspace_refusals(kw, status):
    d = dict(batch=_batch(), heads=4, kv_heads=2, dim=128)
    d.update(kw)
    assert B.lib.prompt_attention_workspace_bytes(ctypes.byref(d["batch"]), d["heads"], d["kv_heads"], d["dim"]) == -1
    assert B.lib.rt_last_error()


def test_null_batch_and_nothing_to_do():
    call = B.lib.prompt_attention_launch
    assert call(None, P, 512, 128, 4, P, 256, 128, P, 256, 128, 2, 128, P, P, 0.1, 0, P, 0, None) == B.RT_ERR_NULL
    assert B.lib.prompt_attention_workspace_bytes(None, 4, 2, 128) == -1
    assert _call(batch=_batch(q_tokens=0), q=None, out=None) == B.RT_OK
    assert _call(batch=_batch(n_seqs=0), q=None, out=None) == B.RT_OK


def test_struct_layouts_match_the_header():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {n: getattr(B, n) for n in ("rt_rotary_spec", "rt_rotary", "rt_rotary_side", "rt_prompt_batch", "rt_compact_batch")}
    lines = [f'printf("%zu\\n", sizeof({n}));' + "".join(f'printf("%zu\\n", offsetof({n}, {f.rstrip(chr(95))}));' for f, _ in t._fields_) for n, t in structs.items()]
    src = '#include <stdio.h>\n#include <stddef.h>\n#include "rmsnorm_tuner.h"\nint main(void){' + "".join(lines) + 'printf("%d\\n", RT_MAX_LAYERS);return 0;}\n'
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "s.c"), "w").write(src)
        subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), os.path.join(d, "s.c"), "-o", os.path.join(d, "s")], check=True)
        got = [int(v) for v in subprocess.run([os.path.join(d, "s")], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for t in structs.values():
        want += [ctypes.sizeof(t)] + [getattr(t, f).offset for f, _ in t._fields_]
    assert got == want + [B.RT_MAX_LAYERS]
