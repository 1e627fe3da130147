"""kv_bounds and kv_select against plain statements of them, bit for bit, and kv_attend_selected against one in 64 bits."""
import math

import pytest
import torch

import mixer_refs as mixers
import operator_refs as refs
from gpu_util import kvx

pytestmark = pytest.mark.gpu

BF16, FP16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
NAN = float("nan")


def normal(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def same_bits(a, b):
    return torch.equal(a.cpu().contiguous().view(torch.uint8), b.cpu().contiguous().view(torch.uint8))


@pytest.fixture(scope="module")
def ctx():
    k = kvx()
    c = k.kv_ctx_create(0)
    yield c
    k.kv_ctx_destroy(c)


class Case:
    """Pages with random rows below every sequence's length and NaN everywhere else, and bounds of nothing yet."""

    def __init__(self, lengths, heads=2, block=16, dim=64, dtype=BF16, nhd=False, pack=1, seed=1):
        self.lengths = list(lengths)
        self.tables, blocks = refs.tables_for(self.lengths, block * pack, seed)
        self.pages = refs.Pages(1, blocks, heads, block, dim, dtype, nhd, pack, seed, fill=NAN)
        rows = normal((2, sum(self.lengths), heads, dim), torch.float32, seed + 1).to(dtype)
        at = 0
        for s, n in enumerate(self.lengths):
            for p in range(n):
                self.pages.put(0, self.tables[s], p, rows[:, at])
                at += 1
        self.upload()

    def upload(self):
        k = kvx()
        p = self.pages
        self.dev = p.data[0].cuda()
        self.pool = k.KvPool.from_tensors([self.dev], p.heads, p.block, k.KVX_LAYOUT_NHD if p.nhd else k.KVX_LAYOUT_HND, p.pack)
        self.batch = k.KvBatch(self.tables.cuda(), ints(self.lengths), max_length=max(self.lengths + [1]))
        self.bounds = k.KvBounds.for_pool(self.pool)
        self.bounds.boxes.fill_(99)
        self.bounds.sizes.fill_(9.0)

    def number(self, s, page):
        return int(self.tables[s, page // self.pages.pack]) * self.pages.pack + page % self.pages.pack

    def page_count(self, s):
        return -(-self.lengths[s] // self.pages.block)

    def want_bounds(self, boxes, sizes, new):
        """boxes and sizes (on the CPU) with those of the last `new` tokens' pages made."""
        for s, n in enumerate(self.lengths):
            for page in range(max(0, n - new) // self.pages.block, self.page_count(s)):
                held = min(self.pages.block, n - page * self.pages.block)
                i = self.number(s, page)
                boxes[i], sizes[i] = mixers.bounds_of(mixers.keys_of(self.pages, 0, self.tables[s], page, held))


def check_bounds(ctx, case, new, stream=None):
    k = kvx()
    boxes, sizes = case.bounds.boxes.cpu().clone(), case.bounds.sizes.cpu().clone()
    case.want_bounds(boxes, sizes, new)
    torch.cuda.synchronize()
    k.kv_bounds(ctx, case.pool, 0, case.batch, case.bounds, new_tokens=new, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(case.bounds.boxes.cpu(), boxes) and torch.equal(case.bounds.sizes.cpu(), sizes)


LENGTHS = [1, 0, 15, 16, 17, 33, 64, 300]


@pytest.mark.parametrize("dtype", [BF16, FP16, E4M3])
@pytest.mark.parametrize("nhd", [False, True])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 256])
def test_bounds(ctx, dtype, nhd, dim):
    case = Case(LENGTHS, heads=3, dim=dim, dtype=dtype, nhd=nhd)
    check_bounds(ctx, case, 300)
    assert kvx().kv_get_device_error(ctx) == -1


@pytest.mark.parametrize("block,pack,new", [(16, 1, 1), (16, 3, 17), (32, 1, 33), (1, 1, 5), (48, 2, 2), (16, 1, 10 ** 9)])
def test_bounds_of_new_tokens_alone(ctx, block, pack, new):
    """Of the pages that hold them, whatever was there; the others' stay."""
    check_bounds(ctx, Case(LENGTHS, block=block, pack=pack), new, stream=torch.cuda.Stream())


@pytest.mark.parametrize("dtype", [BF16, FP16, E4M3])
def test_bounds_of_odd_keys(ctx, dtype):
    """Zeros, one element alone, the smallest and the largest numbers, one sign, infinities and NaN."""
    case = Case([160], heads=1, dtype=dtype)
    put = lambda page, token, value: case.pages.put(0, case.tables[0], page * 16 + token, value.to(dtype).expand(2, 1, 64))
    zero = torch.zeros(64)
    for t in range(16):
        put(0, t, zero)
        put(1, t, zero - 0.0)
        put(2, t, torch.arange(64).float() / 8)
        put(3, t, -torch.arange(64).float() / 8 - 1)
        put(4, t, zero + torch.finfo(dtype).max)
        put(5, t, zero + torch.finfo(dtype).smallest_normal * 2.0 ** -2)
    one = zero.clone()
    one[37] = -3.0
    put(0, 7, one)
    odd = zero.clone()
    odd[63] = NAN
    put(6, 15, odd)
    if dtype != E4M3:
        odd[63] = math.inf
        put(7, 0, odd)
    case.upload()
    check_bounds(ctx, case, 160)


@pytest.mark.parametrize("lengths", [(21, 30, 17, 26), (30, 21, 26, 17), (18, 200, 18, 31), (32, 17, 0, 19)])
@pytest.mark.parametrize("new,pack,many", [(1, 1, False), (40, 3, False), (1, 1, True)])
@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_bounds_of_a_page_that_sequences_hold_to_other_lengths(ctx, lengths, new, pack, many, dtype):
    """Sequences that share their first two pages, the second held to different lengths by each, also by one whose new tokens lie
    further on, and among more sequences than a warp has lanes: bounds of all keys that any of them holds, every time."""
    k = kvx()
    rest = [5] * 70 if many else []
    case = Case([max(lengths)] + rest, block=16, pack=pack, dtype=dtype)
    own = case.tables[:1].repeat(4, 1)
    case.tables = torch.cat([own[:2], case.tables[1:], own[2:]])
    case.lengths = list(lengths[:2]) + rest + list(lengths[2:])
    case.upload()
    boxes, sizes = case.bounds.boxes.cpu().clone(), case.bounds.sizes.cpu().clone()
    case.want_bounds(boxes, sizes, new)
    most = min(32, max(lengths)) - 16
    i = case.number(0, 1)
    boxes[i], sizes[i] = mixers.bounds_of(mixers.keys_of(case.pages, 0, case.tables[0], 1, most))
    if max(lengths) > 32 and new < max(lengths):  # whose first pages are not made for its own sake
        assert any(16 < n <= 32 for n in lengths)
    for _ in range(5):
        case.bounds.boxes.fill_(99)
        case.bounds.sizes.fill_(9.0)
        k.kv_bounds(ctx, case.pool, 0, case.batch, case.bounds, new_tokens=new)
        torch.cuda.synchronize()
        assert torch.equal(case.bounds.boxes.cpu(), boxes) and torch.equal(case.bounds.sizes.cpu(), sizes)


def check_select(ctx, case, q, budget, sinks=1, recent=1, new=1, made=None, stream=None):
    """made: bounds (boxes, sizes) in place of the keys'."""
    k = kvx()
    if made is None:
        k.kv_bounds(ctx, case.pool, 0, case.batch, case.bounds, new_tokens=max(case.lengths + [1]))
    else:
        case.bounds.boxes.copy_(made[0])
        case.bounds.sizes.copy_(made[1])
    torch.cuda.synchronize()
    boxes, sizes = case.bounds.boxes.cpu(), case.bounds.sizes.cpu()
    sel = k.KvSelection(q.shape[1], budget, sinks=sinks, recent=recent, new_tokens=new)
    got = torch.full((len(case.lengths) * new, case.pages.heads, budget), 77, dtype=torch.int32, device="cuda")
    space = k.kv_select_workspace(ctx, case.pool, case.batch, sel)
    space.fill_(0xFF)
    dev = torch.cat([q, q], 1).cuda()[:, :q.shape[1]]
    torch.cuda.synchronize()
    k.kv_select(ctx, case.pool, case.batch, case.bounds, sel, dev, got, space, stream=stream)
    torch.cuda.synchronize()
    got = got.cpu()
    for s, n in enumerate(case.lengths):
        index = [case.number(s, page) for page in range(case.page_count(s))]
        for t in range(new):
            pos = n - new + t
            pages = pos // case.pages.block + 1 if pos >= 0 else 0
            scores = mixers.scores_of(q[s * new + t], boxes[index], sizes[index], case.pages.heads)
            for h in range(case.pages.heads):
                want = mixers.pick(scores[h], pages, budget, sinks, recent)
                assert got[s * new + t, h].tolist() == want + [-1] * (budget - len(want)), (s, t, h)
    return got


LONG = [1, 0, 700, 64, 129, 1500, 33]


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 256])
def test_select(ctx, dtype, cache, dim):
    case = Case(LONG, dim=dim, dtype=cache)
    check_select(ctx, case, normal((len(LONG), 6, dim), dtype, 3), 5)
    assert kvx().kv_get_device_error(ctx) == -1


@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 1), (2, 1, 1), (8, 3, 5), (9, 0, 2), (44, 0, 1), (93, 1, 1), (94, 1, 1), (200, 2, 2)])
def test_budgets_sinks_and_recent_pages(ctx, budget, sinks, recent):
    case = Case(LONG)
    check_select(ctx, case, normal((len(LONG), 2, 64), BF16, 4), budget, sinks, recent)


@pytest.mark.parametrize("group,new", [(1, 4), (3, 2), (8, 9), (16, 4), (17, 64), (33, 2), (64, 1), (65, 3), (128, 2)])
def test_groups_of_heads_and_several_new_tokens(ctx, group, new):
    lengths = [700, 0, 3, 260]
    case = Case(lengths, heads=1)
    check_select(ctx, case, normal((len(lengths) * new, group, 64), FP16, 5), 6, 1, 2, new)


@pytest.mark.parametrize("block,pack", [(16, 3), (32, 1), (1, 1), (48, 2)])
def test_select_over_other_pages(ctx, block, pack):
    case = Case([300, 20, 0, 1000], block=block, pack=pack, nhd=True)
    check_select(ctx, case, normal((4, 4, 64), BF16, 6), 4, stream=torch.cuda.Stream())


def test_equal_scores_go_to_the_lowest_page(ctx):
    """Bounds of few values, so that most scores are equal, and all of them."""
    case = Case([3000, 2000], heads=2)
    g = torch.Generator().manual_seed(7)
    for top in (1, 2):
        boxes = torch.randint(0, top, tuple(case.bounds.boxes.shape), generator=g).to(torch.int8) * 127
        sizes = torch.ones(tuple(case.bounds.sizes.shape))
        for budget in (7, 100):
            check_select(ctx, case, normal((2, 4, 64), BF16, 8), budget, made=(boxes, sizes))


def test_scores_that_are_odd(ctx):
    """Sizes of 0, infinity, NaN and below 0; queries of zeros, infinities and NaN, which count as zeros."""
    case = Case([2000, 2000, 2000, 2000], heads=1)
    boxes = torch.randint(-127, 128, tuple(case.bounds.boxes.shape), generator=torch.Generator().manual_seed(9)).to(torch.int8)
    sizes = normal(tuple(case.bounds.sizes.shape), torch.float32, 10)
    flat = sizes.view(-1)
    flat[3::11], flat[5::13], flat[7::17] = math.inf, NAN, 0.0
    q = normal((4, 2, 64), BF16, 11)
    q[1] = 0
    q[2, 1, 5], q[3, 0, 6] = NAN, math.inf
    check_select(ctx, case, q, 40, made=(boxes, sizes))


def test_keys_that_are_not_finite_are_picked(ctx):
    case = Case([1000], heads=2)
    row = normal((2, 2, 64), BF16, 12)
    row[0, 1, 7] = NAN
    case.pages.put(0, case.tables[0], 400, row)
    case.upload()
    got = check_select(ctx, case, normal((1, 4, 64), BF16, 13), 4)
    assert 25 in got[0, 1].tolist()


def test_missing_pages_come_last_and_are_reported(ctx):
    k = kvx()
    case = Case([200], heads=1)
    q = normal((1, 2, 64), BF16, 14)
    check_select(ctx, case, q, 5)
    case.batch.block_tables[0, 3] = -4
    case.batch.block_tables[0, 6] = 10 ** 6
    sel = k.KvSelection(2, 11, sinks=1, recent=1)
    got = torch.zeros((1, 1, 11), dtype=torch.int32, device="cuda")
    k.kv_select(ctx, case.pool, case.batch, case.bounds, sel, q.cuda(), got, k.kv_select_workspace(ctx, case.pool, case.batch, sel))
    assert got[0, 0].tolist() == [0, 1, 2, 4, 5, 7, 8, 9, 10, 11, 12]
    assert k.kv_get_device_error(ctx) == 3
    before = case.bounds.boxes.clone()
    k.kv_bounds(ctx, case.pool, 0, case.batch, case.bounds, new_tokens=200)
    assert torch.equal(before, case.bounds.boxes)
    assert k.kv_get_device_error(ctx) == 3


def attend(ctx, case, q, selected, new=1, stream=None, **options):
    k = kvx()
    att = k.KvAttention(q.shape[1], new_tokens=new, **options)
    ws = k.kv_attend_selected_workspace(ctx, case.pool, case.batch, att, selected.shape[2], dtype=q.dtype)
    ws.fill_(0xFF)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    dev, sel = q.cuda(), selected.cuda()
    torch.cuda.synchronize()
    k.kv_attend_selected(ctx, case.pool, 0, case.batch, att, sel, dev, out, ws, lse=lse, stream=stream)
    torch.cuda.synchronize()
    return out, lse


def check_attend(ctx, case, q, selected, new=1, missing=(), stream=None, **options):
    scale = options.get("scale") or 1 / math.sqrt(case.pages.dim)
    want, lse, bound, err = mixers.attend_selected(case.pages, 0, case.tables, case.lengths, q, new, selected,
                                                   **{**options, "scale": scale}, missing=missing)
    out, l = attend(ctx, case, q, selected, new, stream, **options)
    off = (out.cpu().double() - want).abs()
    assert bool((off <= bound).all()), f"off by up to {float((off / (bound + 1e-30)).max()):.3g} of the bound"
    assert torch.equal(l.cpu() == -math.inf, lse == -math.inf)
    fine = lse > -math.inf
    assert bool(((l.cpu().double() - lse)[fine].abs() <= err + 1e-6 * lse[fine].abs()).all())
    if not missing:
        assert kvx().kv_get_device_error(ctx) == -1


def some_pages(case, new, budget, seed):
    """Random ascending lists, of which some end early."""
    g = torch.Generator().manual_seed(seed)
    out = torch.full((len(case.lengths) * new, case.pages.heads, budget), -1, dtype=torch.int32)
    for s, n in enumerate(case.lengths):
        for t in range(new):
            pages = max(0, n - new + t) // case.pages.block + 1 if n - new + t >= 0 else 0
            for h in range(case.pages.heads):
                some = torch.randperm(pages, generator=g)[:budget].sort()[0] if pages else torch.zeros(0)
                out[s * new + t, h, :len(some)] = some
    return out


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)])
@pytest.mark.parametrize("nhd", [False, True])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_attend_selected(ctx, dtype, cache, nhd, dim):
    case = Case(LENGTHS, dim=dim, dtype=cache, nhd=nhd)
    scales = {"k_scale": 0.5, "v_scale": 1.75} if cache == E4M3 else {}
    check_attend(ctx, case, normal((len(LENGTHS), 6, dim), dtype, 15), some_pages(case, 1, 3, 16), **scales)


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)])
def test_a_key_that_dominates_gives_its_value(ctx, dtype, cache):
    """Its probability's rounding cancels: the mean is its value, of the type already, but for the others' weights, of
    1e-7 at most, and what 32 bits leave of 64 values below 5: 2^-21 of these."""
    case = Case([64, 64, 64], dtype=cache, seed=23)
    keys = torch.stack([case.pages.rows(0, case.tables[s], range(64)).float() for s in range(3)]).double()  # [seq][2][token][head][dim]
    at = torch.tensor([5, 31, 62])
    chosen = keys[torch.arange(3), :, at]  # [seq][2][head][dim]
    q = (chosen[:, 0].repeat_interleave(3, 1) * torch.tensor([7.0, 8.1, 9.7, 7.3, 11.0, 8.9])[:, None]).to(dtype)
    scores = torch.einsum("shd,sthd->sht", q.double(), keys[:, 0].repeat_interleave(3, 2)) / 8
    weights = scores.softmax(-1)
    assert bool((weights.gather(-1, at[:, None, None].expand(3, 6, 1)) > 1 - 1e-7).all())
    selected = torch.arange(4, dtype=torch.int32).expand(3, 2, 4).contiguous()
    out, _ = attend(ctx, case, q, selected, 1)
    want = chosen[:, 1].repeat_interleave(3, 1)
    assert float(want.abs().max()) < 5
    assert bool(((out.cpu().double() - want).abs() <= 5e-7 + 5 * 2.0 ** -21).all())


@pytest.mark.parametrize("dtype,cache,dim,group", [(BF16, BF16, 128, 4), (FP16, FP16, 96, 2), (BF16, E4M3, 256, 6), (FP16, E4M3, 128, 4),
                                                   (BF16, BF16, 256, 20)])
def test_selected_attention_is_off_by_its_rounding(ctx, dtype, cache, dim, group):
    """Probabilities in two parts are off by 2^-17 of themselves in bf16 and 2^-22 in fp16, scores and sums by some 2^-20: against an
    output's own rounding, 2^-9 / sqrt(3) or 2^-12 / sqrt(3) of it and more in the root mean square, less than 2^-6 of
    that, and 2^-12 of its square.  (Rounded once, a probability is off by as much as an output.)"""
    case = Case([3000, 700, 90], dim=dim, dtype=cache, seed=43)
    q = normal((3, 2 * group, dim), dtype, 44)
    sel = some_pages(case, 1, 60, 45)
    out, _ = attend(ctx, case, q, sel)
    want = mixers.attend_selected(case.pages, 0, case.tables, case.lengths, q, 1, sel, 1 / math.sqrt(dim))[0]
    rounding, off = want.to(dtype).double() - want, out.cpu().double() - want
    assert float(off.square().mean()) <= 1.002 * float(rounding.square().mean())


@pytest.mark.parametrize("cache", [BF16, FP16, E4M3])
@pytest.mark.parametrize("dim,group,new", [(64, 1, 5), (64, 9, 2), (128, 8, 3), (128, 17, 1), (128, 40, 2), (256, 6, 4), (256, 20, 1), (96, 33, 1)])
def test_many_query_rows_and_new_tokens(ctx, cache, dim, group, new):
    lengths = [500, 0, 2, 70]
    case = Case(lengths, dim=dim, dtype=cache, seed=2)
    q = normal((len(lengths) * new, 2 * group, dim), FP16 if cache == FP16 else BF16, 17)
    check_attend(ctx, case, q, some_pages(case, new, 9, 18), new, softcap=20.0)
    check_attend(ctx, case, q, some_pages(case, new, 40, 19), new, scale=0.02, stream=torch.cuda.Stream())


@pytest.mark.parametrize("block,pack", [(16, 3), (32, 1), (1, 1), (48, 2)])
def test_attend_over_other_pages(ctx, block, pack):
    case = Case([300, 20, 0, 1000], block=block, pack=pack)
    check_attend(ctx, case, normal((8, 4, 64), BF16, 20), some_pages(case, 2, 7, 21), 2)


def test_long_lists_are_split_and_joined(ctx):
    case = Case([5000, 1, 2500], heads=1, dim=128)
    check_attend(ctx, case, normal((3, 4, 128), BF16, 22), some_pages(case, 1, 250, 23))


def test_more_sequences_than_a_warp_has_lanes(ctx):
    lengths = [(37 * i) % 200 for i in range(70)]
    case = Case(lengths, heads=1)
    check_attend(ctx, case, normal((140, 2, 64), BF16, 24), some_pages(case, 2, 3, 25), 2)


def test_entries_that_name_no_page_are_left_out(ctx):
    """Negative ones, ones behind the query's page, and ones that do not ascend."""
    case = Case([200, 200, 200], heads=1)
    q = normal((3, 2, 64), BF16, 26)
    sel = torch.tensor([[[-1, 2, 5, 12]], [[1, 13, 40, 2 ** 31 - 1]], [[3, 3, 2, 7]]], dtype=torch.int32)
    sel[0, 0, 0] = -7
    check_attend(ctx, case, q, sel)
    check_attend(ctx, case, q, torch.full((3, 1, 4), -1, dtype=torch.int32))


def test_attend_leaves_missing_pages_out_and_reports_them(ctx):
    case = Case([200], heads=1)
    case.batch.block_tables[0, 2] = -1
    check_attend(ctx, case, normal((1, 2, 64), BF16, 27), torch.tensor([[[0, 2, 5, 12]]], dtype=torch.int32), missing={(0, 2)})
    assert kvx().kv_get_device_error(ctx) == 2


def test_lengths_beyond_the_limit_are_cut_and_reported(ctx):
    k = kvx()
    case = Case([200, 50], heads=1)
    case.batch._c.max_length = 100
    case.lengths[0] = 100
    q = normal((2, 2, 64), BF16, 28)
    out, _ = attend(ctx, case, q, some_pages(case, 1, 4, 29))
    assert k.kv_get_device_error(ctx) == case.tables.shape[1]
    want, _, bound, _ = mixers.attend_selected(case.pages, 0, case.tables, case.lengths, q, 1, some_pages(case, 1, 4, 29), 1 / 8)
    assert bool(((out.cpu().double() - want).abs() <= bound).all())
    check = lambda call: (call(), k.kv_get_device_error(ctx))[1] == case.tables.shape[1]
    sel, got = k.KvSelection(2, 3), torch.zeros((2, 1, 3), dtype=torch.int32, device="cuda")
    assert check(lambda: k.kv_bounds(ctx, case.pool, 0, case.batch, case.bounds, new_tokens=7))
    assert check(lambda: k.kv_select(ctx, case.pool, case.batch, case.bounds, sel, q.cuda(), got, k.kv_select_workspace(ctx, case.pool, case.batch, sel)))


def test_nan_and_infinity_where_a_query_does_not_look(ctx):
    """In pages that are not picked, and behind the query in its own page (NaN there already)."""
    case = Case([100], heads=1)
    sel = torch.tensor([[[1, 4, 6]]], dtype=torch.int32)
    q = normal((1, 2, 64), BF16, 30)
    first = attend(ctx, case, q, sel)
    for p in list(range(16)) + list(range(80, 96)):
        case.pages.put(0, case.tables[0], p, torch.full((2, 1, 64), math.inf, dtype=BF16))
    case.upload()
    assert all(same_bits(a, b) for a, b in zip(first, attend(ctx, case, q, sel)))
    check_attend(ctx, case, q, sel)


def test_captured_run_follows_lengths_and_tables(ctx):
    """Bounds, choice and attention together, replayed as the cache grows, on workspaces of the graph's own."""
    k = kvx()
    case = Case([400, 90], heads=2)
    q = normal((2, 8, 64), BF16, 31).cuda()
    sel, att = k.KvSelection(8, 6, sinks=1, recent=2), k.KvAttention(8)
    picked = torch.zeros((2, 2, 6), dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    case.batch._c.max_length = 400
    spaces = [(k.kv_select_workspace(ctx, case.pool, case.batch, sel), k.kv_attend_selected_workspace(ctx, case.pool, case.batch, att, 6))
              for _ in range(2)]

    def run(space):
        k.kv_bounds(ctx, case.pool, 0, case.batch, case.bounds, new_tokens=400)
        k.kv_select(ctx, case.pool, case.batch, case.bounds, sel, q, picked, space[0])
        k.kv_attend_selected(ctx, case.pool, 0, case.batch, att, picked, q, out, space[1])

    case.batch.lengths.copy_(ints([300, 2]))
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run(spaces[0])
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        run(spaces[0])
    for lengths in ([400, 90], [17, 0], [399, 31]):
        case.batch.lengths.copy_(ints(lengths))
        q.copy_(normal((2, 8, 64), BF16, sum(lengths)))
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), picked.clone()
        out.zero_(), picked.zero_()
        run(spaces[1])
        torch.cuda.synchronize()
        assert same_bits(out, got[0]) and torch.equal(picked, got[1])


def test_a_workspace_that_another_stream_writes_to(ctx):
    """Not allowed, and the picked pages are none in particular, but every call ends, writes its lists alone and nothing but places of
    pages to them; the call that has its workspace to itself again is right.  More pages than a warp's lanes keep."""
    k = kvx()
    pages, budget = 20000, 70
    layer = torch.zeros((pages, 2, 2, 1, 32), dtype=BF16, device="cuda")
    pool = k.KvPool.from_tensors([layer], 2, 1)
    bounds = k.KvBounds.for_pool(pool)
    g = torch.Generator().manual_seed(41)
    bounds.boxes.copy_(torch.randint(-127, 128, tuple(bounds.boxes.shape), generator=g).to(torch.int8).sort(2).values)
    bounds.sizes.copy_(torch.rand(tuple(bounds.sizes.shape), generator=g))
    batch = k.KvBatch(torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1), ints([pages]))
    sel, q = k.KvSelection(4, budget), normal((1, 4, 32), BF16, 42)
    dev, space = q.cuda(), k.kv_select_workspace(ctx, pool, batch, sel)
    room = torch.full((3, 2, budget), -5, dtype=torch.int32, device="cuda")
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(40):
        with torch.cuda.stream(other):
            for _ in range(6):
                space.random_(0, 256)
        k.kv_select(ctx, pool, batch, bounds, sel, dev, room[1:2], space)
    torch.cuda.synchronize()
    assert bool((room[::2] == -5).all()) and bool(((room[1] >= -5) & (room[1] < pages)).all())
    k.kv_select(ctx, pool, batch, bounds, sel, dev, room[1:2], space)
    torch.cuda.synchronize()
    scores = mixers.scores_of(q[0], bounds.boxes.cpu(), bounds.sizes.cpu(), 2)
    for h in range(2):
        assert room[1, h].tolist() == mixers.pick(scores[h], pages, budget, 1, 1)


def test_same_bits_every_time(ctx):
    case = Case([3000, 1, 900], heads=2)
    q = normal((3, 4, 64), BF16, 32)
    sel = some_pages(case, 1, 60, 33)
    runs = [attend(ctx, case, q, sel) for _ in range(3)]
    assert all(same_bits(a, b) for r in runs[1:] for a, b in zip(r, runs[0]))


def test_pages_past_four_gib(ctx):
    """Pages whose byte offset in the layer, and bounds whose offset, need more than 32 bits."""
    k = kvx()
    blocks = (5 << 30) // (2 * 2 * 64 * 2)
    layer = torch.zeros((blocks, 2, 2, 1, 64), dtype=BF16, device="cuda")
    pool = k.KvPool.from_tensors([layer], 2, 1)
    bounds = k.KvBounds.for_pool(pool)
    table = [blocks - 1, 0, blocks - 9, 5, blocks - 2]
    kv, q = normal((5, 4, 64), BF16, 34), normal((1, 4, 64), BF16, 35)
    batch = k.KvBatch(ints([table]), ints([5]))
    k.kv_append(ctx, pool, 0, batch, kv[:, :2].cuda(), kv[:, 2:].cuda(), new_tokens=5)
    k.kv_bounds(ctx, pool, 0, batch, bounds, new_tokens=5)
    sel, att = k.KvSelection(4, 3, sinks=1), k.KvAttention(4)
    picked, out = torch.zeros((1, 2, 3), dtype=torch.int32, device="cuda"), torch.zeros((1, 4, 64), dtype=BF16, device="cuda")
    k.kv_select(ctx, pool, batch, bounds, sel, q.cuda(), picked, k.kv_select_workspace(ctx, pool, batch, sel))
    k.kv_attend_selected(ctx, pool, 0, batch, att, picked, q.cuda(), out, k.kv_attend_selected_workspace(ctx, pool, batch, att, 3))
    small = refs.Pages(1, 5, 2, 1, 64, BF16, fill=0.0)
    boxes, sizes = torch.zeros((5, 2, 2, 64), dtype=torch.int8), torch.zeros((5, 2))
    for p in range(5):
        small.put(0, range(5), p, kv[p].view(2, 2, 64))
        boxes[p], sizes[p] = mixers.bounds_of(kv[p:p + 1, :2])
    assert torch.equal(bounds.boxes[table].cpu(), boxes) and torch.equal(bounds.sizes[table].cpu(), sizes)
    scores = mixers.scores_of(q[0], boxes, sizes, 2)
    assert [picked[0, h].tolist() for h in range(2)] == [mixers.pick(scores[h], 5, 3, 1, 1) for h in range(2)]
    want, _, bound, _ = mixers.attend_selected(small, 0, [range(5)], [5], q, 1, picked.cpu(), 1 / 8)
    assert bool(((out.cpu().double() - want).abs() <= bound).all())


def test_refusals(ctx):
    """Each returns its status before anything is enqueued and leaves the outputs alone."""
    k = kvx()
    case = Case([200, 3], heads=2)
    q = normal((2, 4, 64), BF16, 36).cuda()
    sel, att = k.KvSelection(4, 4), k.KvAttention(4)
    picked = torch.full((2, 2, 4), 77, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 7.0)
    space, room = k.kv_select_workspace(ctx, case.pool, case.batch, sel), k.kv_attend_selected_workspace(ctx, case.pool, case.batch, att, 4)

    def refused(status, f, *a, **kw):
        with pytest.raises(k.KvxError) as e:
            f(*a, **kw)
        assert e.value.status == status, e.value

    def bounds(status, layer=0, bounds=case.bounds, batch=case.batch, **kw):
        refused(status, k.kv_bounds, ctx, case.pool, layer, batch, bounds, **kw)

    bounds(k.KVX_ERANGE, layer=1)
    bounds(k.KVX_EINVAL, new_tokens=0)
    bounds(k.KVX_EINVAL, cache_dtype=E4M3)
    bounds(k.KVX_EDEVICE, bounds=k.KvBounds(case.bounds.boxes.cpu(), case.bounds.sizes.cpu()))
    bounds(k.KVX_ERANGE, batch=k.KvBatch(case.batch.block_tables, case.batch.lengths, max_length=10 ** 6))
    n = case.bounds.boxes.numel()
    odd = torch.zeros(n + 16, dtype=torch.int8, device="cuda")[8:8 + n].view(case.bounds.boxes.shape)
    bounds(k.KVX_EALIGN, bounds=k.KvBounds(odd, case.bounds.sizes))
    with pytest.raises(ValueError):
        k.kv_bounds(ctx, case.pool, 0, case.batch, k.KvBounds(case.bounds.boxes[1:], case.bounds.sizes[1:]))

    def select(status, sel=sel, q=q, picked=picked, space=space, batch=case.batch):
        refused(status, k.kv_select, ctx, case.pool, batch, case.bounds, sel, q, picked, space)

    for bad in (dict(budget=0), dict(budget=4, sinks=-1), dict(budget=4, recent=0), dict(budget=4, sinks=3, recent=2)):
        select(k.KVX_EINVAL, sel=k.KvSelection(4, **bad), picked=picked[..., :bad["budget"]].contiguous())
    select(k.KVX_EINVAL, sel=k.KvSelection(3, 4), q=q[:, :3])
    select(k.KVX_EINVAL, sel=k.KvSelection(4, 4, new_tokens=65), q=q.repeat(65, 1, 1), picked=picked.repeat(65, 1, 1))
    select(k.KVX_EINVAL, sel=k.KvSelection(258, 4), q=torch.zeros((2, 258, 64), dtype=BF16, device="cuda"))
    select(k.KVX_ERANGE, space=space[:16])
    select(k.KVX_EALIGN, space=torch.zeros(space.numel() + 16, dtype=torch.uint8, device="cuda")[4:])
    select(k.KVX_EALIGN, q=torch.zeros((2, 4, 72), dtype=BF16, device="cuda")[..., 4:68])
    select(k.KVX_EDEVICE, q=q.cpu())
    select(k.KVX_EDEVICE, picked=picked.cpu())
    with pytest.raises(ValueError):
        k.kv_select(ctx, case.pool, case.batch, case.bounds, sel, q, picked[..., :3].contiguous(), space)
    with pytest.raises(TypeError):
        k.kv_select(ctx, case.pool, case.batch, case.bounds, sel, q, picked.long(), space)
    with pytest.raises(TypeError):
        k.kv_select(ctx, case.pool, case.batch, case.bounds, sel, q.float(), picked, space)

    def attends(status, att=att, q=q, out=out, picked=picked, room=room, layer=0, **kw):
        refused(status, k.kv_attend_selected, ctx, case.pool, layer, case.batch, att, picked, q, out, room, **kw)

    attends(k.KVX_EINVAL, att=k.KvAttention(4, window=5))
    attends(k.KVX_EINVAL, att=k.KvAttention(4, slopes=torch.ones(4, device="cuda")))
    attends(k.KVX_EINVAL, att=k.KvAttention(4, softcap=-1.0))
    attends(k.KVX_EINVAL, picked=picked[..., :0].contiguous())
    attends(k.KVX_ERANGE, room=room[:16])
    attends(k.KVX_ERANGE, layer=-1)
    attends(k.KVX_EINVAL, q=q.half(), out=out.half())
    attends(k.KVX_EDEVICE, picked=picked.cpu())
    attends(k.KVX_EDEVICE, out=out.cpu())
    with pytest.raises(ValueError):
        k.kv_attend_selected(ctx, case.pool, 0, case.batch, att, picked[:1], q, out, room)
    many = k.KvBatch(torch.zeros((65535, 4), dtype=torch.int32, device="cuda"), torch.zeros(65535, dtype=torch.int32, device="cuda"))
    refused(k.KVX_ERANGE, k.kv_attend_selected_workspace, ctx, case.pool, many, k.KvAttention(4096, new_tokens=64), 4)
    k.kv_fault_inject("launch")
    select(k.KVX_ECUDA)
    torch.cuda.synchronize()
    assert bool((out == 7.0).all()) and bool((picked == 77).all()) and bool((case.bounds.boxes == 99).all())
    assert k.kv_get_device_error(ctx) == -1


def test_nothing_to_do(ctx):
    k = kvx()
    case = Case([3], heads=1)
    empty = k.KvBatch(torch.zeros((0, 4), dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"))
    q, picked = torch.zeros((0, 2, 64), dtype=BF16, device="cuda"), torch.zeros((0, 1, 4), dtype=torch.int32, device="cuda")
    sel, att = k.KvSelection(2, 4), k.KvAttention(2)
    before = k.kv_ctx_stats(ctx)["kernel_launches"]
    k.kv_bounds(ctx, case.pool, 0, empty, case.bounds)
    k.kv_select(ctx, case.pool, empty, case.bounds, sel, q, picked, k.kv_select_workspace(ctx, case.pool, empty, sel))
    k.kv_attend_selected(ctx, case.pool, 0, empty, att, picked, q, q, k.kv_attend_selected_workspace(ctx, case.pool, empty, att, 4))
    assert k.kv_ctx_stats(ctx)["kernel_launches"] == before
