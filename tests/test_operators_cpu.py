"""The operators' entry points without a GPU: no context, no call; and the plain statements that the GPU tests
compare with, held against worked values and against differences."""
import ctypes
import math

import pytest
import torch

import operator_refs as refs
from paper_2609_15021_gb300 import kvxfer as k


def test_no_context_is_refused_before_any_cuda_call():
    pool, batch = k.kvx_pool(), k.kvx_batch()
    r = ctypes.byref
    out = ctypes.c_int64()
    assert k._lib.kv_append(None, r(pool), 0, r(batch), r(k.kvx_new_rows()), 0, 0, None) == k.KVX_EINVAL
    assert k._lib.kv_attend(None, r(pool), 0, r(batch), r(k.kvx_attention()), 0, 0, 0, 0, None) == k.KVX_EINVAL
    assert k._lib.kv_attend_workspace(None, r(pool), r(batch), r(k.kvx_attention()), r(out)) == k.KVX_EINVAL
    assert k._lib.kv_evict(None, r(pool), r(batch), r(k.kvx_eviction()), None) == k.KVX_EINVAL
    state, sb = k.kvx_state(), k.kvx_state_batch()
    assert k._lib.kv_state_conv(None, r(state), r(sb), r(k.kvx_conv()), 0, 0, None) == k.KVX_EINVAL
    assert k._lib.kv_state_scan(None, r(state), r(sb), r(k.kvx_scan()), 0, 0, 0, 0, 0, 0, 0, None) == k.KVX_EINVAL
    assert k._lib.kv_state_scan_workspace(None, r(sb), r(k.kvx_scan()), r(out)) == k.KVX_EINVAL


def test_bindings_structures_match_the_header(tmp_path):
    """Sizes and offsets of the structures, as a C compiler lays them out."""
    import os
    import subprocess
    names = ["kvx_batch", "kvx_new_rows", "kvx_attention", "kvx_eviction", "kvx_state", "kvx_state_batch", "kvx_conv", "kvx_scan"]
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "kvxfer.h"', "int main(void) {"]
    for n in names:
        lines.append(f'  printf("{n} %zu\\n", sizeof({n}));')
        for f in getattr(k, n)._fields_:
            lines.append(f'  printf("{n}.{f[0]} %zu\\n", offsetof({n}, {f[0]}));')
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["  return 0;", "}"]))
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run(["gcc", "-I", include, str(src), "-o", str(tmp_path / "layout")], check=True)
    said = dict(l.split() for l in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.splitlines())
    for n in names:
        assert int(said[n]) == ctypes.sizeof(getattr(k, n))
        for f in getattr(k, n)._fields_:
            assert int(said[f"{n}.{f[0]}"]) == getattr(getattr(k, n), f[0]).offset, (n, f[0])


def test_binding_refuses_other_types_and_shapes():
    t, n = torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        k.KvBatch(t.long(), n)
    with pytest.raises(ValueError):
        k.KvBatch(t, n[:1])
    with pytest.raises(ValueError):
        k.KvBatch(t.T, n.repeat(2)[:3])
    with pytest.raises(TypeError):
        k.KvAttention(2, slopes=torch.zeros(2, dtype=torch.float64))
    with pytest.raises(TypeError):
        k._type_of(torch.float32)
    with pytest.raises(ValueError):
        k.StateSlots(torch.zeros(100, dtype=torch.uint8), 2, 64)


def test_scale_of_zero_is_not_the_default():
    """0 is how the C call marks the default, so the binding must not pass a caller's 0 on."""
    with pytest.raises(ValueError):
        k.KvAttention(2, scale=0.0)
    assert k.KvAttention(2)._c.scale == 0.0 and k.KvAttention(2, scale=0.5)._c.scale == 0.5


def test_reference_attention_by_hand():
    """Two keys, scores 0 and log 3: probabilities 1/4 and 3/4."""
    pages = refs.Pages(1, 1, 1, 4, 8, torch.bfloat16, fill=0.0)
    rows = torch.zeros((2, 1, 8))
    rows[1, 0, 0] = 4.0
    pages.put(0, [0], 0, rows.to(torch.bfloat16))
    rows[0, 0, 1], rows[1, 0, 0] = 1.0, 8.0
    pages.put(0, [0], 1, rows.to(torch.bfloat16))
    q = torch.zeros((1, 1, 8), dtype=torch.bfloat16)
    q[0, 0, 1] = 1.0
    out, lse, w, bound, err = refs.attend(pages, 0, [[0]], [2], q, 1, math.log(3.0))
    assert abs(float(out[0, 0, 0]) - 7.0) < 1e-12
    assert abs(float(lse[0, 0]) - math.log(4.0)) < 1e-12
    assert torch.allclose(w[0, 0], torch.tensor([0.25, 0.75], dtype=torch.float64))


def test_reference_selection_by_hand():
    w = [0.5, 0.1, math.nan, 0.5, 0.9, 0.1, 0.2]
    assert refs.select(w, 7, 4, 1, 1) == [0, 3, 4, 6]
    assert refs.select(w, 7, 3, 0, 0) == [0, 3, 4]
    assert refs.select(w, 3, 5, 1, 1) == [0, 1, 2]
    assert refs.select(w, 7, 6, 0, 0) == [0, 1, 3, 4, 5, 6]


def test_reference_scan_is_the_recurrence_in_closed_form():
    """out_t = sum_s (C_t . B_s) exp(sum of the exponents between) d_s x_s."""
    g = torch.Generator().manual_seed(1)
    x, b, c = (torch.randn((7, 1, 8), generator=g, dtype=torch.float64) for _ in range(3))
    dt, A = torch.rand((7, 1), generator=g, dtype=torch.float64), torch.tensor([-0.7], dtype=torch.float64)
    out, state, _, _ = refs.scan(x, dt, A, b, c, None, None, False, torch.zeros((1, 8, 8), dtype=torch.float64))
    for t in range(7):
        want = sum((c[t, 0] @ b[s, 0]) * torch.exp(A * dt[s + 1:t + 1].sum()) * dt[s] * x[s, 0] for s in range(t + 1))
        assert torch.allclose(out[t, 0], want)
