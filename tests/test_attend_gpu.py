"""kv_append and kv_attend against plain 64-bit statements of them."""
import math

import pytest
import torch

import operator_refs as refs
from gpu_util import kvx

pytestmark = pytest.mark.gpu

BF16, FP16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
NAN = float("nan")


def normal(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


@pytest.fixture(scope="module")
def ctx():
    k = kvx()
    c = k.kv_ctx_create(0)
    yield c
    k.kv_ctx_destroy(c)


class Case:
    """Pages with random rows below every sequence's length and NaN everywhere else."""

    def __init__(self, lengths, heads=2, block=16, dim=64, dtype=BF16, nhd=False, pack=1, seed=1, layers=1):
        k = kvx()
        self.lengths = list(lengths)
        self.tables, blocks = refs.tables_for(self.lengths, block * pack, seed)
        self.pages = refs.Pages(layers, blocks, heads, block, dim, dtype, nhd, pack, seed, fill=NAN)
        for l in range(layers):
            for s, n in enumerate(self.lengths):
                for p in range(n):
                    self.pages.put(l, self.tables[s], p, normal((2, heads, dim), torch.float32, seed * 7919 + s * 4099 + p).to(dtype))
        self.upload()

    def upload(self):
        k = kvx()
        p = self.pages
        self.dev = [x.cuda() for x in p.data]
        self.pool = k.KvPool.from_tensors(self.dev, p.heads, p.block, k.KVX_LAYOUT_NHD if p.nhd else k.KVX_LAYOUT_HND, p.pack)
        self.batch = k.KvBatch(self.tables.cuda(), torch.tensor(self.lengths, dtype=torch.int32, device="cuda"),
                               max_length=max(self.lengths + [1]))


def same_bits(a, b):
    return torch.equal(a.cpu().contiguous().view(torch.uint8), b.cpu().contiguous().view(torch.uint8))


def run_attend(ctx, case, q, new=1, weights=None, lse=True, stream=None, workspace=None, **options):
    k = kvx()
    att = k.KvAttention(q.shape[1], new_tokens=new, **options)
    ws = workspace if workspace is not None else k.kv_attend_workspace(ctx, case.pool, case.batch, att,
                                                                       weights=weights is not None, dtype=q.dtype)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    l = torch.full(q.shape[:2], 7.0, device="cuda") if lse else None
    k.kv_attend(ctx, case.pool, 0, case.batch, att, q.cuda(), out, ws, lse=l, weights=weights, stream=stream)
    torch.cuda.synchronize()
    return out, l


def check_attend(ctx, case, q, new=1, with_weights=False, **options):
    slopes = options.get("slopes")
    ref = dict(options)
    scale = ref.pop("scale", None) or 1 / math.sqrt(case.pages.dim)
    want, lse, w, bound, err = refs.attend(case.pages, 0, case.tables, case.lengths, q, new, scale,
                                           **{**ref, "slopes": None if slopes is None else slopes.cpu()})
    weights = None
    if with_weights:
        weights = torch.full((len(case.lengths), case.pages.heads, w.shape[-1] + 3), 0.25, device="cuda")
    out, l = run_attend(ctx, case, q, new, weights=weights, **options)
    off = (out.cpu().double() - want).abs()
    assert bool((off <= bound).all()), f"off by up to {float((off / (bound + 1e-30)).max()):.3g} of the bound"
    assert torch.equal(l.cpu() == -math.inf, lse == -math.inf)
    fine = lse > -math.inf
    assert bool(((l.cpu().double() - lse)[fine].abs() <= err + 1e-6 * lse[fine].abs()).all())
    if with_weights:
        got = weights.cpu().double()
        rows = q.shape[1] // case.pages.heads * new
        assert bool(((got[..., :w.shape[-1]] - 0.25 - w).abs() <= w * 2 * err + 2.0 ** -23 * (rows + 1)).all())
        for s, n in enumerate(case.lengths):
            assert bool((got[s, :, n:] == 0.25).all())
    assert kvx().kv_get_device_error(ctx) == -1
    return out


# lengths around a step's 16 keys, around pages, of one token, of none, and long enough to be split
LENGTHS = [1, 0, 15, 16, 17, 33, 64, 300]


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)])
@pytest.mark.parametrize("nhd", [False, True])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_types_layouts_and_rows(ctx, dtype, cache, nhd, dim):
    case = Case(LENGTHS, heads=2, dim=dim, dtype=cache, nhd=nhd)
    scales = {"k_scale": 0.5, "v_scale": 1.75} if cache == E4M3 else {}
    check_attend(ctx, case, normal((len(LENGTHS), 6, dim), dtype, 3), with_weights=True, **scales)


@pytest.mark.parametrize("group", [1, 2, 5, 8, 16, 17, 33])
@pytest.mark.parametrize("new", [1, 2, 5])
def test_groups_of_heads_and_several_new_tokens(ctx, group, new):
    lengths = [0, 1, 3, 31, 200]  # the first ones are shorter than the new tokens: rows without a key
    case = Case(lengths, heads=2, dim=64)
    check_attend(ctx, case, normal((len(lengths) * new, 2 * group, 64), BF16, 4), new, with_weights=True)


# rows of queries (heads of a group x new tokens) that take two, three or four tiles of eight, and blocks of them
ROWS = [(5, 2), (6, 4), (8, 4), (11, 4), (40, 1)]


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("group,new", ROWS)
def test_many_query_rows(ctx, dtype, cache, dim, group, new):
    lengths = [0, 1, 3, 17, 64, 210]
    case = Case(lengths, heads=2, dim=dim, dtype=cache, seed=2)
    scales = {"k_scale": 0.5, "v_scale": 1.75} if cache == E4M3 else {}
    check_attend(ctx, case, normal((len(lengths) * new, 2 * group, dim), dtype, 29), new, with_weights=True, **scales)


@pytest.mark.parametrize("cache", [BF16, FP16, E4M3])
@pytest.mark.parametrize("dim,group,new", [(64, 6, 4), (128, 3, 4), (128, 8, 4), (256, 4, 4), (256, 6, 4)])
def test_many_query_rows_of_long_caches_with_cap_bias_and_window(ctx, cache, dim, group, new):
    """Split over the cache and joined."""
    case = Case([2500, 700, 9], heads=1, dim=dim, dtype=cache, block=32, seed=3)
    q = normal((3 * new, group, dim), FP16 if cache == FP16 else BF16, 30)
    slopes = torch.exp2(-torch.arange(1, group + 1, device="cuda").float())
    check_attend(ctx, case, q, new, with_weights=True, softcap=20.0, slopes=slopes)
    check_attend(ctx, case, q, new, with_weights=True, window=600)


@pytest.mark.parametrize("cache", [BF16, FP16, E4M3])
@pytest.mark.parametrize("dim,group", [(64, 1), (64, 4), (64, 8), (128, 1), (128, 4), (128, 8), (256, 1), (256, 4), (256, 6)])
def test_values_that_are_not_finite_in_every_form(ctx, cache, dim, group):
    """As test_nan_and_infinity_where_a_row_does_not_look, for each type, head size and number of tiles."""
    new = 4
    case = Case([30, 64], heads=1, dim=dim, dtype=cache)
    for s, n in enumerate(case.lengths):
        case.pages.put(0, case.tables[s], n - 1, torch.tensor([NAN, math.inf]).to(cache).view(2, 1, 1).expand(2, 1, dim))
        case.pages.put(0, case.tables[s], n - 12, torch.tensor([math.inf, NAN]).to(cache).view(2, 1, 1).expand(2, 1, dim))
    case.upload()
    q = normal((2 * new, group, dim), FP16 if cache == FP16 else BF16, 13)
    weights = torch.zeros((2, 1, 64), device="cuda")
    out, lse = run_attend(ctx, case, q, new, weights=weights, window=9)
    want, l, _, bound, err = refs.attend(case.pages, 0, case.tables, case.lengths, q, new, 1 / math.sqrt(dim), window=9)
    for s in range(2):
        for t in range(1, new - 1):  # position n-4+t: sees n-12+t .. n-4+t
            row = s * new + t
            assert bool(((out[row].cpu().double() - want[row]).abs() <= bound[row]).all())
            assert bool(((lse[row].cpu().double() - l[row]).abs() <= err + 1e-6).all())
        assert bool(torch.isnan(out[s * new + new - 1]).all())


def test_scores_beyond_the_range_of_fp16(ctx):
    """Scores are kept in 32 bits: those of fp16 queries and keys may pass 65,504."""
    case = Case([1, 50, 400], heads=1, dim=64, dtype=FP16)
    q = normal((3, 2, 64), FP16, 8, 5000.0)
    check_attend(ctx, case, q, scale=1.5)
    _, lse, _, _, _ = refs.attend(case.pages, 0, case.tables, case.lengths, q, 1, 1.5)
    assert float(lse.max()) > 65504


@pytest.mark.parametrize("block,pack,dim,cache", [(1, 1, 64, BF16), (3, 5, 64, BF16), (32, 49, 64, E4M3),
                                                  (8, 1, 72, FP16), (48, 2, 80, BF16), (16, 1, 16, E4M3), (16, 1, 8, BF16)])
def test_pages_that_end_inside_a_step(ctx, block, pack, dim, cache):
    case = Case([1, 47, 130], heads=1, block=block, dim=dim, dtype=cache, pack=pack)
    check_attend(ctx, case, normal((3, 4, dim), FP16 if cache == FP16 else BF16, 5), with_weights=True)


@pytest.mark.parametrize("window", [1, 2, 16, 40, 1000])
@pytest.mark.parametrize("new", [1, 3])
def test_window(ctx, window, new):
    case = Case([0, 1, 17, 100, 260], heads=2)
    check_attend(ctx, case, normal((5 * new, 4, 64), BF16, 6), new, with_weights=True, window=window)


@pytest.mark.parametrize("window", [261, 2 ** 30, 2 ** 31 - 4, 2 ** 31 - 1])
def test_window_of_more_than_every_key(ctx, window):
    """As no window at all, also where a sequence is shorter than its new tokens, and whatever the workspace holds."""
    k = kvx()
    case = Case([1, 2, 0, 5, 260], heads=2)
    q = normal((20, 4, 64), BF16, 27)
    att = k.KvAttention(4, new_tokens=4, window=window)
    ws = k.kv_attend_workspace(ctx, case.pool, case.batch, att, weights=True)
    ws.fill_(0x7F)
    weights, plain = torch.zeros((5, 2, 260), device="cuda"), torch.zeros((5, 2, 260), device="cuda")
    got = run_attend(ctx, case, q, 4, weights=weights, workspace=ws, window=window)
    want = run_attend(ctx, case, q, 4, weights=plain)
    assert all(same_bits(a, b) for a, b in zip(got + (weights,), want + (plain,)))
    check_attend(ctx, case, q, 4, with_weights=True, window=window)


@pytest.mark.parametrize("softcap,slopes,scale", [(30.0, False, None), (5.0, False, 1.5), (0.0, True, None), (20.0, True, 0.3)])
def test_cap_bias_and_scale(ctx, softcap, slopes, scale):
    case = Case([1, 90, 513], heads=2, dim=128)
    s = torch.exp2(-torch.arange(1, 7, device="cuda").float()) if slopes else None
    check_attend(ctx, case, normal((6, 6, 128), BF16, 7, 3.0), 2, with_weights=True, softcap=softcap, slopes=s, scale=scale)


def test_large_scores_do_not_overflow(ctx):
    case = Case([1, 50, 400], heads=1, dim=64)
    check_attend(ctx, case, normal((3, 2, 64), BF16, 8, 100.0))


@pytest.mark.parametrize("seqs", [1, 3, 40])
def test_long_sequences_are_split_and_joined(ctx, seqs):
    lengths = [3000 - 61 * i for i in range(min(seqs, 3))] + [5 + i for i in range(seqs - 3)]
    case = Case(lengths, heads=1, dim=64, block=64)
    check_attend(ctx, case, normal((seqs, 4, 64), BF16, 9), with_weights=True)


def test_rows_of_a_projection_and_other_strides(ctx):
    """q, k, v as slices of one projection's output, out in [head][token] order; append then attend."""
    k = kvx()
    lengths, new, h, hq, d = [5, 2, 40], 2, 2, 4, 64
    case = Case(lengths, heads=h, dim=d)
    qkv = normal((3 * new, hq + 2 * h, d), BF16, 10)
    dev = qkv.cuda()
    k.kv_append(ctx, case.pool, 0, case.batch, dev[:, hq:hq + h], dev[:, hq + h:], new_tokens=new)
    for s, n in enumerate(lengths):
        for i in range(new):
            case.pages.put(0, case.tables[s], n - new + i, torch.stack([qkv[s * new + i, hq:hq + h], qkv[s * new + i, hq + h:]]))
    assert same_bits(case.dev[0], case.pages.data[0])
    want, _, _, bound, _ = refs.attend(case.pages, 0, case.tables, lengths, qkv[:, :hq], new, 1 / 8)
    att = k.KvAttention(hq, new_tokens=new)
    ws = k.kv_attend_workspace(ctx, case.pool, case.batch, att)
    out = torch.zeros((hq, 3 * new, d), dtype=BF16, device="cuda")
    k.kv_attend(ctx, case.pool, 0, case.batch, att, dev[:, :hq], out.transpose(0, 1), ws)
    torch.cuda.synchronize()
    assert bool(((out.transpose(0, 1).cpu().double() - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)])
@pytest.mark.parametrize("nhd", [False, True])
@pytest.mark.parametrize("dim", [8, 48, 128, 256])
def test_append_of_prompts(ctx, dtype, cache, nhd, dim):
    if cache == E4M3 and dim % 16:
        pytest.skip("a row is a multiple of 16 bytes")
    k = kvx()
    new, before = [0, 1, 37, 5, 16], [7, 0, 3, 0, 16]
    lengths = [a + b for a, b in zip(new, before)]
    case = Case(lengths, heads=3, dim=dim, dtype=cache, nhd=nhd, block=8, pack=3)
    starts = [sum(new[:i]) for i in range(len(new) + 1)]
    kv = normal((starts[-1], 6, dim), dtype, 11, 300.0 if cache == E4M3 else 1.0)
    kv[0, 0, :5] = torch.tensor([math.inf, -math.inf, NAN, 1e-9, -0.0])
    scales = (1.7, 0.3) if cache == E4M3 else (1.0, 1.0)
    dev = kv.cuda()
    k.kv_append(ctx, case.pool, 0, case.batch, dev[:, :3], dev[:, 3:], starts=torch.tensor(starts, dtype=torch.int32, device="cuda"),
                k_scale=scales[0], v_scale=scales[1])
    torch.cuda.synchronize()
    for s, n in enumerate(lengths):
        for i in range(new[s]):
            rows = kv[starts[s] + i].view(2, 3, dim)
            if cache == E4M3:
                rows = torch.stack([refs.quantise(rows[j], scales[j]) for j in range(2)])
            case.pages.put(0, case.tables[s], n - new[s] + i, rows)
    got, want = case.dev[0].cpu(), case.pages.data[0]
    if cache == E4M3:  # a NaN keeps no sign
        assert torch.equal(torch.nan_to_num(got.float(), nan=1e4), torch.nan_to_num(want.float(), nan=1e4))
    else:
        assert same_bits(got, want)
    assert k.kv_get_device_error(ctx) == -1


@pytest.mark.parametrize("scale", [2.0 ** -126, 2.0 ** -100, 2.0 ** 120, 3.0e38])
def test_append_with_scales_at_the_ends_of_the_range(ctx, scale):
    """Zeros stay zeros and other values are their quotients, or the nearest that 8 bits hold."""
    k = kvx()
    case = Case([4], heads=1, dim=64, dtype=E4M3)
    kv = normal((4, 2, 64), BF16, 28)
    kv[:, :, :16], kv[:, :, 16:32] = 0.0, (kv[:, :, 16:32].float() * min(scale, 1e37)).to(BF16)
    k.kv_append(ctx, case.pool, 0, case.batch, kv[:, :1].cuda(), kv[:, 1:].cuda(), new_tokens=4, k_scale=scale, v_scale=scale)
    torch.cuda.synchronize()
    for i in range(4):
        case.pages.put(0, case.tables[0], i, refs.quantise(kv[i].view(2, 1, 64), scale))
    got, want = case.dev[0].cpu().float(), case.pages.data[0].float()
    assert torch.equal(torch.nan_to_num(got, nan=1e4), torch.nan_to_num(want, nan=1e4))


@pytest.mark.parametrize("scale", [1e-39, 1e-45])
def test_append_refuses_scales_that_have_no_reciprocal(ctx, scale):
    k = kvx()
    case = Case([2], heads=1, dim=64, dtype=E4M3)
    kv = torch.zeros((2, 1, 64), dtype=BF16, device="cuda")
    for which in ("k_scale", "v_scale"):
        with pytest.raises(k.KvxError) as e:
            k.kv_append(ctx, case.pool, 0, case.batch, kv, kv, new_tokens=2, **{which: scale})
        assert e.value.status == k.KVX_EINVAL
    torch.cuda.synchronize()
    assert same_bits(case.dev[0], case.pages.data[0])


def test_append_drops_rows_before_the_first_position(ctx):
    k = kvx()
    case = Case([2, 0], heads=1, dim=64)
    kv = normal((8, 2, 64), BF16, 12)
    k.kv_append(ctx, case.pool, 0, case.batch, kv[:, :1].cuda(), kv[:, 1:].cuda(), new_tokens=4)
    torch.cuda.synchronize()
    for i in range(2):
        case.pages.put(0, case.tables[0], i, kv[2 + i].view(2, 1, 64))
    assert same_bits(case.dev[0], case.pages.data[0])


def test_nan_and_infinity_where_a_row_does_not_look(ctx):
    """A draft token's K and V are not finite: the rows before it, which do not see it, are as without it, and so
    are rows whose window it has left."""
    new = 4
    case = Case([30, 64], heads=1, dim=64)
    for s, n in enumerate(case.lengths):
        case.pages.put(0, case.tables[s], n - 1, torch.tensor([NAN, math.inf]).to(BF16).view(2, 1, 1).expand(2, 1, 64))
        case.pages.put(0, case.tables[s], n - 12, torch.tensor([math.inf, NAN]).to(BF16).view(2, 1, 1).expand(2, 1, 64))
    case.upload()
    q = normal((2 * new, 3, 64), BF16, 13)
    out, lse = run_attend(ctx, case, q, new, window=9)
    want, l, _, bound, err = refs.attend(case.pages, 0, case.tables, case.lengths, q, new, 1 / 8, window=9)
    for s in range(2):
        for t in range(1, new - 1):  # position n-4+t: sees n-12+t .. n-4+t
            row = s * new + t
            assert bool(((out[row].cpu().double() - want[row]).abs() <= bound[row]).all())
            assert bool(((lse[row].cpu().double() - l[row]).abs() <= err + 1e-6).all())
        assert bool(torch.isnan(out[s * new + new - 1]).all())


def test_missing_pages_are_left_out_and_reported(ctx):
    k = kvx()
    case = Case([200, 90], heads=2)
    case.tables[0, 3], case.tables[1, 0] = -1, 10 ** 6
    case.batch = k.KvBatch(case.tables.cuda(), case.batch.lengths, max_length=200)
    q = normal((2, 4, 64), BF16, 14)
    want, lse, w, bound, err = refs.attend(case.pages, 0, case.tables, case.lengths, q, 1, 1 / 8, missing={(0, 3), (1, 0)})
    weights = torch.zeros((2, 2, 200), device="cuda")
    out, l = run_attend(ctx, case, q, weights=weights)
    assert bool(((out.cpu().double() - want).abs() <= bound).all())
    assert bool(((l.cpu().double() - lse).abs() <= err + 1e-6).all())
    assert bool(((weights.cpu().double() - w).abs() <= w * 2 * err + 1e-6).all())
    assert k.kv_get_device_error(ctx) == 0
    assert k.kv_get_device_error(ctx) == -1


def test_lengths_beyond_the_limit_are_cut_and_reported(ctx):
    k = kvx()
    case = Case([64, 20], heads=1)
    q = normal((2, 2, 64), BF16, 15)
    want, _, _, bound, _ = refs.attend(case.pages, 0, case.tables, [40, 0], q, 1, 1 / 8)
    case.batch = k.KvBatch(case.tables.cuda(), torch.tensor([1 << 30, -5], dtype=torch.int32, device="cuda"), max_length=40)
    out, _ = run_attend(ctx, case, q)
    assert bool(((out.cpu().double() - want).abs() <= bound).all())
    assert k.kv_get_device_error(ctx) == case.tables.shape[1]


def test_captured_call_follows_lengths_and_tables(ctx):
    """A captured append + attend, replayed with other lengths, tables, queries and rows."""
    k = kvx()
    case = Case([33, 5], heads=2)
    qkv = normal((2, 8, 64), BF16, 16).cuda()
    att = k.KvAttention(4)
    batch = k.KvBatch(case.batch.block_tables, case.batch.lengths)
    ws = k.kv_attend_workspace(ctx, case.pool, batch, att, weights=True)
    weights = torch.zeros((2, 2, case.tables.shape[1] * 16), device="cuda")
    out = torch.zeros((2, 4, 64), dtype=BF16, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        k.kv_append(ctx, case.pool, 0, batch, qkv[:, 4:6], qkv[:, 6:])
        k.kv_attend(ctx, case.pool, 0, batch, att, qkv[:, :4], out, ws, weights=weights)
    for seed, lengths in ((17, [33, 5]), (18, [20, 0]), (19, [1, 4])):
        new = normal((2, 8, 64), BF16, seed)
        qkv.copy_(new)
        weights.zero_()
        case.batch.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for s, n in enumerate(lengths):
            if n:
                case.pages.put(0, case.tables[s], n - 1, torch.stack([new[s, 4:6], new[s, 6:]]))
        want, _, w, bound, err = refs.attend(case.pages, 0, case.tables, lengths, new[:, :4], 1, 1 / 8)
        assert bool(((out.cpu().double() - want).abs() <= bound).all())
        assert bool(((weights.cpu().double()[..., :w.shape[-1]] - w).abs() <= w * 2 * err + 1e-6).all())
    assert k.kv_get_device_error(ctx) == -1


def test_same_bits_every_time_and_on_another_stream(ctx):
    case = Case([3000, 700, 1], heads=2, dim=128, block=32)
    q = normal((3, 8, 128), BF16, 20)
    stream = torch.cuda.Stream()
    runs = []
    for st in (None, stream, None):
        weights = torch.zeros((3, 2, 3000), device="cuda")
        torch.cuda.synchronize()
        out, lse = run_attend(ctx, case, q, weights=weights, stream=st)
        runs.append((out, lse, weights))
    for r in runs[1:]:
        assert all(same_bits(a, b) for a, b in zip(r, runs[0]))


def test_one_workspace_serves_call_after_call(ctx):
    """Batches of other shapes in between leave the workspace fit for the next call."""
    k = kvx()
    big, small = Case([2000, 900], heads=2), Case([1, 0, 60], heads=1)
    qb, qs = normal((2, 4, 64), BF16, 21), normal((3, 16, 64), BF16, 22)
    att = k.KvAttention(4)
    need = [k.kv_attend_workspace(ctx, c.pool, c.batch, k.KvAttention(h), weights=True).numel()
            for c, h in ((big, 4), (small, 16))]
    ws = torch.zeros(max(need), dtype=torch.uint8, device="cuda")
    outs = []
    for _ in range(3):
        outs.append((run_attend(ctx, big, qb, workspace=ws)[0], run_attend(ctx, small, qs, workspace=ws)[0]))
    assert all(same_bits(a, b) for o in outs[1:] for a, b in zip(o, outs[0]))
    want, _, _, bound, _ = refs.attend(big.pages, 0, big.tables, big.lengths, qb, 1, 1 / 8)
    assert bool(((outs[2][0].cpu().double() - want).abs() <= bound).all())


def test_pages_past_four_gib(ctx):
    """Pages whose byte offset in the layer needs more than 32 bits."""
    k = kvx()
    blocks = (5 << 30) // (2 * 16 * 128 * 2)
    layer = torch.zeros((blocks, 2, 1, 16, 128), dtype=BF16, device="cuda")
    pool = k.KvPool.from_tensors([layer], 1, 16)
    pages = [blocks - 1, 0, blocks - 9]
    tables = torch.tensor([pages], dtype=torch.int32, device="cuda")
    kv, q = normal((40, 2, 128), BF16, 23), normal((1, 8, 128), BF16, 24)
    batch = k.KvBatch(tables, torch.tensor([40], dtype=torch.int32, device="cuda"))
    k.kv_append(ctx, pool, 0, batch, kv[:, :1].cuda(), kv[:, 1:].cuda(), new_tokens=40)
    att = k.KvAttention(8)
    out = torch.zeros((1, 8, 128), dtype=BF16, device="cuda")
    k.kv_attend(ctx, pool, 0, batch, att, q.cuda(), out, k.kv_attend_workspace(ctx, pool, batch, att))
    torch.cuda.synchronize()
    small = refs.Pages(1, 3, 1, 16, 128, BF16, fill=0.0)
    for p in range(40):
        small.put(0, [0, 1, 2], p, kv[p].view(2, 1, 128))
    assert same_bits(layer[pages], small.data[0])
    want, _, _, bound, _ = refs.attend(small, 0, [[0, 1, 2]], [40], q, 1, 1 / math.sqrt(128))
    assert bool(((out.cpu().double() - want).abs() <= bound).all())


def test_refusals(ctx):
    """Each returns its status before anything is enqueued and leaves the outputs alone."""
    k = kvx()
    case = Case([20, 3], heads=2)
    q = normal((2, 4, 64), BF16, 25).cuda()
    out, att = torch.full_like(q, 7.0), k.KvAttention(4)
    ws = k.kv_attend_workspace(ctx, case.pool, case.batch, att, weights=True)
    kv = torch.zeros((2, 2, 64), dtype=BF16, device="cuda")

    def attend(status, q=q, out=out, att=att, layer=0, batch=case.batch, ws=ws, **kw):
        with pytest.raises(k.KvxError) as e:
            k.kv_attend(ctx, case.pool, layer, batch, att, q, out, ws, **kw)
        assert e.value.status == status, e.value

    attend(k.KVX_ERANGE, layer=1)
    attend(k.KVX_EINVAL, att=k.KvAttention(3), q=q[:, :3], out=out[:, :3])
    attend(k.KVX_EINVAL, att=k.KvAttention(4, new_tokens=65), q=q.repeat(65, 1, 1), out=out.repeat(65, 1, 1))
    attend(k.KVX_EINVAL, att=k.KvAttention(4, softcap=NAN))
    attend(k.KVX_EINVAL, att=k.KvAttention(4, scale=math.inf))
    attend(k.KVX_EINVAL, att=k.KvAttention(4, window=-1))
    attend(k.KVX_EINVAL, q=q.half(), out=out.half())  # a bf16 cache
    attend(k.KVX_EINVAL, out=torch.zeros((1, 4, 64), dtype=BF16, device="cuda").expand(2, 4, 64))
    wide = torch.zeros((2, 4, 72), dtype=BF16, device="cuda")
    attend(k.KVX_EALIGN, q=wide[..., 4:68])
    attend(k.KVX_EDEVICE, q=q.cpu())
    attend(k.KVX_EDEVICE, out=out.cpu())
    attend(k.KVX_ERANGE, batch=k.KvBatch(case.batch.block_tables, case.batch.lengths, max_length=10 ** 6))
    attend(k.KVX_ERANGE, ws=ws[:16], weights=torch.zeros((2, 2, 20), device="cuda"))
    assert bool((out == 7.0).all())
    for bad in ({"query": q[:1]}, {"lse": torch.zeros((2, 3), device="cuda")}, {"weights": torch.zeros((2, 2, 19), device="cuda")}):
        with pytest.raises(ValueError):
            k.kv_attend(ctx, case.pool, 0, case.batch, att, **{"query": q, "out": out, "workspace": ws, **bad})
    with pytest.raises(TypeError):
        k.kv_attend(ctx, case.pool, 0, case.batch, att, q, out.half(), ws)
    with pytest.raises(TypeError):
        k.KvBatch(case.tables.cuda().long(), case.batch.lengths)

    def append(status, key=kv, layer=0, **kw):
        with pytest.raises(k.KvxError) as e:
            k.kv_append(ctx, case.pool, layer, case.batch, key, key, **kw)
        assert e.value.status == status, e.value

    append(k.KVX_ERANGE, layer=-1)
    append(k.KVX_EINVAL, key=kv.half())
    append(k.KVX_EINVAL, k_scale=-1.0)
    append(k.KVX_EINVAL, v_scale=math.inf)
    append(k.KVX_EDEVICE, key=kv.cpu())
    append(k.KVX_EALIGN, key=torch.zeros((2, 2, 68), dtype=BF16, device="cuda")[..., :64])
    assert same_bits(case.dev[0], case.pages.data[0])
    k.kv_fault_inject("launch")
    append(k.KVX_ECUDA)
    assert k.kv_get_device_error(ctx) == -1


@pytest.mark.parametrize("stride", [2 ** 60, 2 ** 61, 2 ** 62, 2 ** 63 - 1])
def test_table_strides_beyond_64_bits_of_bytes(ctx, stride):
    """Their products with the sequences must not wrap into a small extent."""
    k = kvx()
    case = Case([20, 3, 1, 0, 5], heads=2)
    case.batch._c.table_stride = stride
    q = normal((5, 4, 64), BF16, 25).cuda()
    out, ws = torch.full_like(q, 7.0), torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    with pytest.raises(k.KvxError) as e:
        k.kv_attend(ctx, case.pool, 0, case.batch, k.KvAttention(4), q, out, ws)
    assert e.value.status == k.KVX_EINVAL
    with pytest.raises(k.KvxError) as e:
        k.kv_append(ctx, case.pool, 0, case.batch, q[:, :2], q[:, 2:])
    assert e.value.status == k.KVX_EINVAL
    torch.cuda.synchronize()
    assert bool((out == 7.0).all()) and same_bits(case.dev[0], case.pages.data[0])


def test_more_rows_than_a_launch_has(ctx):
    """65,535 sequences of 64 tokens and 4,096 heads are 1.7e10 rows of queries: refused, not wrapped."""
    k = kvx()
    case = Case([3], heads=1)
    many = k.KvBatch(torch.zeros((65535, 4), dtype=torch.int32, device="cuda"),
                     torch.zeros(65535, dtype=torch.int32, device="cuda"))
    with pytest.raises(k.KvxError) as e:
        k.kv_attend_workspace(ctx, case.pool, many, k.KvAttention(4096, new_tokens=64))
    assert e.value.status == k.KVX_ERANGE


@pytest.mark.parametrize("byte", [0x00, 0xFF, 0x7F])
def test_workspace_needs_no_initial_contents(ctx, byte):
    k = kvx()
    case = Case([500, 1, 0, 37], heads=2)
    q = normal((4 * 3, 8, 64), BF16, 26).cuda()
    att = k.KvAttention(8, new_tokens=3)

    def once(fill):
        ws = k.kv_attend_workspace(ctx, case.pool, case.batch, att, weights=True)
        ws.view(torch.uint8).fill_(fill)
        out, weights = torch.full_like(q, 7.0), torch.zeros((4, 2, 500), device="cuda")
        lse = torch.zeros((12, 8), device="cuda")
        k.kv_attend(ctx, case.pool, 0, case.batch, att, q, out, ws, lse=lse, weights=weights)
        return out, weights, lse

    for got, want in zip(once(byte), once(0x3C)):
        assert same_bits(got, want)


def test_nothing_to_do(ctx):
    k = kvx()
    case = Case([3], heads=1)
    empty = k.KvBatch(torch.zeros((0, 4), dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"))
    q = torch.zeros((0, 2, 64), dtype=BF16, device="cuda")
    att = k.KvAttention(2)
    before = k.kv_ctx_stats(ctx)["kernel_launches"]
    k.kv_attend(ctx, case.pool, 0, empty, att, q, q, k.kv_attend_workspace(ctx, case.pool, empty, att))
    k.kv_append(ctx, case.pool, 0, empty, q[:, :1], q[:, :1])
    assert k.kv_ctx_stats(ctx)["kernel_launches"] == before
