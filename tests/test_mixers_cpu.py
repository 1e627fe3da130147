"""The rotated append, the choice of pages and the delta rule without a GPU: refusals before any CUDA call, the binding's
checks and structures, and the plain statements that the GPU tests compare with, held against worked values."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

import mixer_refs as refs
import operator_refs
from paper_2609_15021_gb300 import kvxfer as k


def test_no_context_is_refused_before_any_cuda_call():
    pool, batch, state, sb = k.kvx_pool(), k.kvx_batch(), k.kvx_state(), k.kvx_state_batch()
    r, out = ctypes.byref, ctypes.c_int64()
    assert k._lib.kv_append_rotary(None, r(pool), 0, r(batch), r(k.kvx_new_rows()), r(k.kvx_rotary()), 0, 0, 0, 0, None) == k.KVX_EINVAL
    assert k._lib.kv_bounds(None, r(pool), 0, r(batch), 0, 1, r(k.kvx_bounds()), None) == k.KVX_EINVAL
    assert k._lib.kv_select_workspace(None, r(pool), r(batch), r(k.kvx_selection()), r(out)) == k.KVX_EINVAL
    assert k._lib.kv_select(None, r(pool), r(batch), r(k.kvx_bounds()), r(k.kvx_selection()), 0, 0, 0, 0, None) == k.KVX_EINVAL
    assert k._lib.kv_attend_selected_workspace(None, r(pool), r(batch), r(k.kvx_attention()), 1, r(out)) == k.KVX_EINVAL
    assert k._lib.kv_attend_selected(None, r(pool), 0, r(batch), r(k.kvx_attention()), 1, 0, 0, 0, 0, 0, None) == k.KVX_EINVAL
    assert k._lib.kv_state_delta_workspace(None, r(sb), r(k.kvx_delta()), r(out)) == k.KVX_EINVAL
    assert k._lib.kv_state_delta(None, r(state), r(sb), r(k.kvx_delta()), 0, 0, 0, 0, 0, 0, 0, 0, None) == k.KVX_EINVAL


def test_bindings_structures_match_the_header(tmp_path):
    """Sizes and offsets of the structures, as a C compiler lays them out."""
    names = ["kvx_rotary", "kvx_bounds", "kvx_selection", "kvx_delta"]
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
    freq = torch.ones(4)
    with pytest.raises(TypeError):
        k.KvRotary(2, freq.double())
    with pytest.raises(ValueError):
        k.KvRotary(2, freq.view(2, 2))
    with pytest.raises(ValueError):
        k.KvRotary(2, freq, q_weight=freq.view(2, 2))
    with pytest.raises(ValueError):
        k.KvRotary(2, freq, k_weight=torch.ones(8)[::2])
    with pytest.raises(ValueError):  # the C call's mark for 1
        k.KvRotary(2, freq, scale=0.0)
    boxes, sizes = torch.zeros((3, 2, 2, 64), dtype=torch.int8), torch.zeros((3, 2))
    with pytest.raises(TypeError):
        k.KvBounds(boxes.int(), sizes)
    with pytest.raises(TypeError):
        k.KvBounds(boxes, sizes.double())
    with pytest.raises(ValueError):
        k.KvBounds(boxes, sizes[:2])
    with pytest.raises(ValueError):
        k.KvBounds(boxes[:, :, :1], sizes)
    with pytest.raises(ValueError):
        k.KvBounds(boxes[::2], sizes[::2])


def test_rotation_by_hand():
    """A quarter turn of the first pair, none of the second."""
    x = torch.tensor([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    freq = torch.tensor([math.pi / 6, 0.0])
    got, size = refs.rotate(x, [3], freq, True, 1.0, None, 0.0, 0.0)
    assert torch.allclose(got[0, 0], torch.tensor([-2.0, 1.0, 3.0, 4.0, 5.0], dtype=torch.float64), atol=1e-6)
    assert size[0, 0].tolist() == [3.0, 3.0, 7.0, 7.0, 5.0]
    got, _ = refs.rotate(x, [3], freq, False, 2.0, None, 0.0, 0.0)
    assert torch.allclose(got[0, 0], torch.tensor([-6.0, 4.0, 2.0, 8.0, 5.0], dtype=torch.float64), atol=1e-6)
    got, _ = refs.rotate(x, [0], None, False, 1.0, torch.tensor([0.0, 1.0, 1.0, 1.0, 1.0]), 0.0, 1.0)
    assert torch.allclose(got[0, 0, :2], torch.tensor([1.0, 4.0], dtype=torch.float64) / math.sqrt(11.0))


def test_bounds_hold_every_key_and_scores_every_product():
    """A page's score is no less than the rounded query's product with any of its keys."""
    g = torch.Generator().manual_seed(1)
    keys = torch.randn((16, 2, 64), generator=g).to(torch.bfloat16)
    box, size = refs.bounds_of(keys)
    k64 = keys.double()
    by = size.double()[:, None]
    assert bool((box[:, 0].double() * by <= k64.amin(0) + 1e-6).all()) and bool((box[:, 1].double() * by >= k64.amax(0) - 1e-6).all())
    q = torch.randn((4, 64), generator=g)
    score = refs.scores_of(q, box[None], size[None], 2)
    step = q.abs().amax(-1, keepdim=True) / 127
    whole = (torch.round(q / step) * step).double()
    for h in range(2):
        most = (whole[2 * h:2 * h + 2] @ k64[:, h].T).max()
        assert float(score[h, 0]) >= float(most) - 1e-5
    assert refs.bounds_of(torch.zeros((3, 1, 8)))[1].tolist() == [0.0]
    odd = keys.clone()
    odd[3, 1, 5] = math.nan
    box, size = refs.bounds_of(odd)
    assert box[1, 0].tolist() == [-127] * 64 and float(size[1]) > 1e38 and float(size[0]) < 1.0


def test_pick_by_hand():
    s = [0.5, 0.1, math.nan, 0.5, 0.9, 0.1, 0.2, 0.0]
    assert refs.pick(s, 8, 4, 1, 1) == [0, 3, 4, 7]
    assert refs.pick(s, 8, 3, 0, 1) == [0, 4, 7]
    assert refs.pick(s, 4, 4, 0, 1) == [0, 1, 2, 3]
    assert refs.pick(s, 7, 2, 1, 1) == [0, 6]
    assert refs.pick(s, 7, 6, 0, 1) == [0, 1, 3, 4, 5, 6]


def test_selected_attention_over_all_pages_is_the_attention():
    pages = operator_refs.Pages(1, 6, 2, 16, 32, torch.bfloat16, seed=3)
    tables = [[3, 1, 5], [0, 2, 4]]
    q = torch.randn((4, 4, 32), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    want, lse, _, _, _ = operator_refs.attend(pages, 0, tables, [40, 1], q, 2, 0.3, softcap=5.0)
    every = torch.arange(3, dtype=torch.int32).expand(4, 2, 3)
    out, l, _, _ = refs.attend_selected(pages, 0, tables, [40, 1], q, 2, every, 0.3, softcap=5.0)
    assert torch.allclose(out, want) and torch.allclose(l, lse)


def test_delta_rule_writes_what_a_key_reads():
    """Orthonormal keys, full steps, no decay: the state maps each key to its last value."""
    keys = torch.eye(8, dtype=torch.float64)[[0, 3, 0]].view(3, 1, 8)
    v = torch.tensor([[1.0, 2.0], [3.0, 4.0], [5.0, 6.0]], dtype=torch.float64).view(3, 1, 2)
    out, state, _, _, _ = refs.delta(keys, keys, v, torch.ones((3, 1)), torch.zeros((1, 2, 8)), sigmoid=False, normalize=False, scale=1.0)
    assert torch.allclose(out[:, 0], v[:, 0])
    want = torch.zeros((2, 8), dtype=torch.float64)
    want[:, 0], want[:, 3] = v[2, 0], v[1, 0]
    assert torch.allclose(state[0], want)


def test_delta_rule_is_its_product_of_matrices():
    """S_T = sum over s of b_s v_s k_s^T times the products of a_t (I - b_t k_t k_t^T) behind s."""
    g = torch.Generator().manual_seed(5)
    t_n, n, p = 6, 8, 4
    q, k64 = (torch.randn((t_n, 1, n), generator=g, dtype=torch.float64) for _ in range(2))
    v = torch.randn((t_n, 1, p), generator=g, dtype=torch.float64)
    beta, dt = (torch.randn((t_n, 1), generator=g, dtype=torch.float64) for _ in range(2))
    A, first = torch.tensor([-0.7], dtype=torch.float64), torch.randn((1, p, n), generator=g, dtype=torch.float64)
    _, state, _, _, _ = refs.delta(q, k64, v, beta, first, dt, A, torch.tensor([0.3]))
    unit = k64[:, 0] / torch.sqrt((k64[:, 0] ** 2).sum(-1, keepdim=True) + 1e-6)
    b, a = torch.sigmoid(beta[:, 0]), torch.exp(A * torch.nn.functional.softplus(dt[:, 0] + torch.tensor(0.3, dtype=torch.float32).double()))
    step = [a[t] * (torch.eye(n, dtype=torch.float64) - b[t] * torch.outer(unit[t], unit[t])) for t in range(t_n)]
    want = first[0]
    for t in range(t_n):
        want = want @ step[t] + b[t] * torch.outer(v[t, 0], unit[t])
    assert torch.allclose(state[0], want, atol=1e-9)


SEARCH = r"""
#include <algorithm>
#include <cstdio>
#include <vector>
#include "pick_border.cuh"
using namespace kvx;
static uint64_t state = 12345;
static uint32_t any() { return (uint32_t)((state = state * 6364136223846793005ull + 1442695040888963407ull) >> 32); }
#define NEED(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

// The kernel's search; `change` makes other ranks between passes.
template <class F>
static int search(std::vector<uint32_t>& ranks, Border& b, F change, int* passes) {
  bool ended = false;
  for (*passes = 0; *passes < kPickPasses && !ended; ++*passes) {
    std::vector<int> counts(kPickBins);
    const int shift = b.shift();
    NEED(b.low <= b.high && shift <= 32 - kPickBits);
    for (uint32_t r : ranks)
      if (r >= b.low && r <= b.high) {
        NEED((r - b.low) >> shift < (uint32_t)kPickBins);
        ++counts[(r - b.low) >> shift];
      }
    int bin = kPickBins - 1, left = b.want;
    while (bin >= 0 && left > counts[bin]) left -= counts[bin--];
    ended = !b.narrow(shift, bin < 0 ? 0xDEADBEEFu : (uint32_t)bin, bin < 0 ? 0 : left, bin < 0 ? 0x7FFFFFFF : counts[bin]);
    change();
  }
  NEED(ended);
  return 0;
}

int main() {
  const int sizes[] = {1, 2, 5, 100, 4097, 9000};
  for (int n : sizes)
    for (uint32_t span : {0u, 1u, 2046u, 2047u, 2048u, 1u << 21, 0xFFFFFFFEu})
      for (int k = 0; k < 20; ++k) {
        std::vector<uint32_t> ranks(n);
        auto make = [&] { const uint32_t base = 1 + any() % (0xFFFFFFFFu - span); for (uint32_t& r : ranks) r = base + (uint32_t)(any() * (uint64_t)span >> 32); };
        make();
        std::vector<uint32_t> sorted = ranks;
        std::sort(sorted.begin(), sorted.end());
        const int32_t want = 1 + any() % n;
        int passes;
        Border b = {sorted.front(), sorted.back(), want};
        if (search(ranks, b, [] {}, &passes)) return 1;
        // those above the border and the first `equal` at it are the want largest
        const uint32_t last = sorted[n - want];
        const long above = sorted.end() - std::upper_bound(sorted.begin(), sorted.end(), b.rank);
        NEED(above + b.equal == want && (b.equal ? b.rank == last : b.rank < last));
        // ranks of other calls between the passes, among them none within what is searched
        Border other = {sorted.front(), sorted.back(), want};
        if (search(ranks, other, make, &passes)) return 1;
        make();
        Border none = {sorted.front(), sorted.back(), want};
        if (search(ranks, none, [&] { std::fill(ranks.begin(), ranks.end(), 0u); }, &passes)) return 1;
        NEED(passes <= kPickPasses);
      }
  printf("ok\n");
}
"""


def test_search_for_the_last_picked_page_ends(tmp_path):
    """The search's arithmetic as the kernel has it: three passes at most, with the right border where the ranks stay, and an end
    where another call writes to the workspace between two passes."""
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_15021_gb300", "csrc")
    src = tmp_path / "search.cpp"
    src.write_text(SEARCH)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", csrc, str(src), "-o", str(tmp_path / "search")], check=True)
    done = subprocess.run([str(tmp_path / "search")], capture_output=True, text=True, timeout=60)
    assert done.returncode == 0 and done.stdout == "ok\n", done.stdout


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_bounds_miss_a_key_by_no_more_than_they_say(dtype):
    """A size and a quotient are each off by 2^-24 of themselves at most, so bounds times sizes miss a key by 2^-24 of the largest,
    and a score the rounded rows' largest product by as much of its terms for each of the bounds and its two products; some do
    miss.  A page with a key that is not finite has the largest score, and no query but zeros or odd ones gives every page 0."""
    g = torch.Generator().manual_seed(2)
    unit, missed = 2.0 ** -24, 0
    for scale in (1.0, 3e-3, 700.0, 1e-38 if dtype is torch.bfloat16 else 1e-6):
        keys = (torch.randn((40, 16, 2, 64), generator=g) * scale).to(dtype)
        boxes, sizes = (torch.stack(x) for x in zip(*(refs.bounds_of(k_) for k_ in keys)))
        by, k64 = sizes.double()[:, :, None], keys.double()
        low, high = boxes[:, :, 0].double() * by, boxes[:, :, 1].double() * by
        slack = unit * k64.abs().amax((1, 3))[:, :, None] + 2.0 ** -143
        assert bool((low <= k64.amin(1) + slack).all()) and bool((high >= k64.amax(1) - slack).all())
        missed += int((low > k64.amin(1)).sum()) + int((high < k64.amax(1)).sum())
        q = torch.randn((4, 64), generator=g)
        score = refs.scores_of(q, boxes, sizes, 2).double()
        step = (q.abs().amax(-1, keepdim=True) / 127).double()
        rows = torch.round(q / step.float()).double() * step
        for h in range(2):
            most = torch.einsum("rd,ptd->prt", rows[2 * h:2 * h + 2], k64[:, :, h]).amax((1, 2))
            terms = rows[2 * h:2 * h + 2].abs().sum(-1).max() * k64[:, :, h].abs().amax((1, 2))
            assert bool((score[h] >= most - 4 * unit * terms - 2.0 ** -130).all())
    assert missed > 0
    odd = keys.clone()
    odd[7, 3, 0, 9] = math.nan
    boxes, sizes = (torch.stack(x) for x in zip(*(refs.bounds_of(k_) for k_ in odd)))
    assert int(refs.scores_of(torch.randn((2, 64), generator=g), boxes, sizes, 2)[0].argmax()) == 7
    for q in (torch.zeros((2, 64)), torch.full((2, 64), math.nan)):
        scores = refs.scores_of(q, boxes, sizes, 2)
        assert not bool(scores.any()) and refs.pick(scores[0], 40, 3, 0, 1) == [0, 1, 39]
