"""kv_append_rotary against a plain 64-bit statement of it."""
import math

import pytest
import torch

import mixer_refs as mixers
import operator_refs as refs
from gpu_util import kvx

pytestmark = pytest.mark.gpu

BF16, FP16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def normal(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module")
def ctx():
    k = kvx()
    c = k.kv_ctx_create(0)
    yield c
    k.kv_ctx_destroy(c)


class Step:
    """Pages of a few sequences with rows of their own, and a step's new rows within one projection's output."""

    def __init__(self, lengths, new, heads=2, q_heads=4, dim=64, block=16, dtype=BF16, cache=None, nhd=False, pack=1, seed=1,
                 spare=0, scale=2.0):
        k = kvx()
        self.lengths, self.new, self.dtype, self.q_heads = list(lengths), list(new), dtype, q_heads
        self.tables, blocks = refs.tables_for(self.lengths, block * pack, seed)
        self.pages = refs.Pages(1, blocks, heads, block, dim, cache or dtype, nhd, pack, seed)
        self.starts = [spare + sum(new[:i]) for i in range(len(new) + 1)]  # rows in front of the first and behind the last are nobody's
        self.rows = self.starts[-1] + spare
        self.qkv = normal((self.rows, q_heads + 2 * heads, dim), dtype, seed + 1, scale)
        self.dev = self.pages.data[0].cuda()
        self.pool = k.KvPool.from_tensors([self.dev], heads, block, k.KVX_LAYOUT_NHD if nhd else k.KVX_LAYOUT_HND, pack)
        self.batch = k.KvBatch(self.tables.cuda(), ints(self.lengths), max_length=max(self.lengths + [1]))

    def owner(self):
        """(row, sequence, place in its cache) of every row that has an owner."""
        for s, n in enumerate(self.new):
            for i in range(n):
                yield self.starts[s] + i, s, self.lengths[s] - n + i


def check(ctx, st, freq, interleaved=False, weights=(None, None), eps=1e-6, offset=0.0, scale=1.0, positions=None, scales=(1.0, 1.0),
          in_place=False, stream=None, single=False, missing=()):
    k = kvx()
    h, hq, d = st.pages.heads, st.q_heads, st.pages.dim
    qkv = st.qkv.cuda()
    q, key, value = qkv[:, :hq], qkv[:, hq:hq + h], qkv[:, hq + h:]
    wide = torch.full((st.rows, hq + 1, d), 7.0, dtype=st.dtype, device="cuda")
    out = q if in_place else wide[:, :hq]
    before = out.cpu().clone()
    inv_freq = None if freq is None else freq.cuda()
    rotary = k.KvRotary(hq, inv_freq, interleaved=interleaved, scale=scale, q_weight=None if weights[0] is None else weights[0].cuda(),
                        k_weight=None if weights[1] is None else weights[1].cuda(), eps=eps, weight_offset=offset)
    torch.cuda.synchronize()
    kw = {"new_tokens": st.new[0]} if single else {"starts": ints(st.starts)}
    k.kv_append_rotary(ctx, st.pool, 0, st.batch, rotary, q, key, value, out, k_scale=scales[0], v_scale=scales[1],
                       positions=None if positions is None else ints(positions), stream=stream, **kw)
    torch.cuda.synchronize()
    places = {row: p for row, _, p in st.owner()}
    at = [positions[r] if positions is not None else places.get(r, 0) for r in range(st.rows)]
    x = st.qkv
    unit = refs.UNIT[st.dtype]
    got = out.cpu().double()
    want, size = mixers.rotate(x[:, :hq], at, freq, interleaved, scale, weights[0], eps, offset)
    # A norm is a sum of at most 256 squares in 32 bits and a reciprocal root, a factor 1 + 2^-19; an angle's turn in 32
    # bits is off by 2^-25 of a turn, sine and cosine by less than 2^-21; products and a sum; then one rounding.
    bound = unit * want.abs() + 2.0 ** -18 * size + 2.0 ** -25
    for r in range(st.rows):
        if r in places:
            assert bool(((got[r] - want[r]).abs() <= bound[r]).all()), (r, float(((got[r] - want[r]).abs() / bound[r]).max()))
        else:
            assert torch.equal(out.cpu()[r], before[r])
    assert bool((wide[:, hq:] == 7.0).all())
    keys, ksize = mixers.rotate(x[:, hq:hq + h], at, freq, interleaved, scale, weights[1], eps, offset)
    expect = st.pages.data.clone()
    st.pages.data = st.dev.cpu()[None]
    for r, s, p in st.owner():
        if p < 0 or (s, p // (st.pages.block * st.pages.pack)) in missing:
            continue
        k_row, v_row = st.pages.rows(0, st.tables[s], [p])[:, 0]
        if st.pages.dtype == E4M3:
            want_v = refs.quantise(x[r, hq + h:], scales[1])
            y, slack = keys[r] / scales[0], ksize[r] / scales[0]
            off = (k_row.double() - y.clamp(-448, 448)).abs()
            # the nearest of 4 significant bits, or of multiples of 2^-9
            limit = 2.0 ** -4 * y.abs().clamp(max=448) + 2.0 ** -10 + 2.0 ** -17 * slack
        else:
            want_v = x[r, hq + h:]
            off, limit = (k_row.double() - keys[r]).abs(), unit * keys[r].abs() + 2.0 ** -18 * ksize[r] + 2.0 ** -25
        assert torch.equal(v_row.view(torch.uint8), want_v.contiguous().view(torch.uint8))
        assert bool((off <= limit).all()), (r, float((off / limit).max()))
        kept = refs.Pages.__new__(refs.Pages)
        kept.__dict__.update(st.pages.__dict__, data=expect)
        kept.put(0, st.tables[s], p, torch.stack([k_row, v_row]))
    assert torch.equal(expect.view(torch.uint8), st.pages.data.view(torch.uint8))  # nothing else has changed
    if not missing:
        assert k.kv_get_device_error(ctx) == -1


def frequencies(half, base=10000.0):
    return (base ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).float()


NEW, LENGTHS = [1, 0, 3, 17, 40], [1, 5, 35, 17, 300]


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)])
@pytest.mark.parametrize("nhd", [False, True])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 256])
def test_types_layouts_and_rows(ctx, dtype, cache, nhd, dim):
    for interleaved in (False, True):
        st = Step(LENGTHS, NEW, dim=dim, dtype=dtype, cache=cache, nhd=nhd, q_heads=6, spare=3)
        weights = [normal((dim,), dtype, 7 + i, 0.1) + 1 for i in range(2)]
        check(ctx, st, frequencies(dim // 2), interleaved, weights, scales=(0.5, 1.75) if cache == E4M3 else (1.0, 1.0))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rotary", [(64, 0), (64, 2), (64, 16), (64, 20), (64, 48), (96, 30), (128, 32), (128, 126), (256, 64), (256, 200)])
def test_part_of_the_head_is_rotated(ctx, interleaved, dim, rotary):
    """Halves that are whole vectors of eight and that are not."""
    for in_place in (False, True):
        st = Step(LENGTHS, NEW, dim=dim, q_heads=3, heads=1)
        check(ctx, st, frequencies(rotary // 2) if rotary else None, interleaved, (normal((dim,), BF16, 8), normal((dim,), BF16, 9)),
              in_place=in_place)


@pytest.mark.parametrize("which", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norms_of_queries_or_keys_alone(ctx, which, interleaved):
    st = Step(LENGTHS, NEW, dim=96)
    weights = [normal((96,), BF16, 10 + i, 0.1) if w else None for i, w in enumerate(which)]
    check(ctx, st, frequencies(24), interleaved, weights, eps=1e-3, offset=1.0, scale=0.75)


@pytest.mark.parametrize("heads,q_heads", [(1, 1), (1, 71), (8, 64), (3, 9)])
@pytest.mark.parametrize("tokens", [1, 700])
def test_heads_and_many_tokens(ctx, heads, q_heads, tokens):
    st = Step([tokens + 20], [tokens], heads=heads, q_heads=q_heads, dim=64, dtype=FP16)
    check(ctx, st, frequencies(32), False, [normal((64,), FP16, 3, 0.1) + 1] * 2)


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_warp_a_token_and_a_warp_a_unit_give_the_same_bits(ctx, interleaved):
    """A call of few tokens an SM and one of many share their rows: what becomes of a row does not depend on the others."""
    k = kvx()
    few = 4 * torch.cuda.get_device_properties(0).multi_processor_count
    rotary = k.KvRotary(4, frequencies(32).cuda(), interleaved=interleaved, q_weight=normal((64,), BF16, 6, 0.1).cuda(),
                        k_weight=normal((64,), BF16, 7, 0.1).cuda())
    for dtype, cache in ((BF16, BF16), (BF16, E4M3)):
        got = []
        for rows in (few, few + 1):
            st = Step([few + 1], [few + 1], dtype=dtype, cache=cache)
            batch = k.KvBatch(st.tables.cuda(), ints([rows]), max_length=few + 1)
            qkv, out = st.qkv.cuda()[:rows], torch.zeros((rows, 4, 64), dtype=dtype, device="cuda")
            k.kv_append_rotary(ctx, st.pool, 0, batch, rotary, qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], out, new_tokens=rows)
            st.pages.data = st.dev.cpu()[None]
            got.append((out[:few].view(torch.int16).cpu(), st.pages.rows(0, st.tables[0], range(few)).view(torch.uint8)))
        assert all(torch.equal(a, b) for a, b in zip(*got))


def test_more_sequences_than_a_warp_has_lanes(ctx):
    new = [i % 4 for i in range(75)]
    st = Step([n + 7 * i for i, n in enumerate(new)], new, spare=2)
    check(ctx, st, frequencies(32), True)


def test_one_token_of_every_sequence(ctx):
    st = Step([1, 16, 17, 200], [1] * 4)
    check(ctx, st, frequencies(32), single=True)
    st = Step([3, 16, 17, 200], [3] * 4)
    check(ctx, st, frequencies(32), single=True, stream=torch.cuda.Stream())


def test_positions_of_their_own(ctx):
    """Positions that ran ahead of an evicted cache's, up to the largest there are, and negative ones."""
    st = Step(LENGTHS, NEW, spare=1)
    positions = [(i * 104729 * 397) % (2 ** 31) for i in range(st.rows)]
    positions[1], positions[2], positions[3] = 2 ** 31 - 1, -5, -2 ** 31
    check(ctx, st, frequencies(32), False, positions=positions)
    check(ctx, Step(LENGTHS, NEW, spare=1), frequencies(32), True, positions=positions)


def test_rows_before_the_first_position_are_rotated_and_dropped(ctx):
    st = Step([2, 0, 30], [4, 2, 3])
    check(ctx, st, frequencies(32), False)


@pytest.mark.parametrize("block,pack", [(16, 3), (32, 1), (1, 1), (48, 2)])
def test_pages_and_blocks(ctx, block, pack):
    check(ctx, Step(LENGTHS, NEW, block=block, pack=pack, cache=E4M3), frequencies(32))


def test_small_and_large_rows_and_scales(ctx):
    """Rows whose squares leave 16 bits but not 32, and e4m3's clamp and least numbers."""
    for size in (1e-4, 1e3):
        st = Step(LENGTHS, NEW, dtype=FP16, scale=size)
        check(ctx, st, frequencies(32), False, [normal((64,), FP16, 3, 0.1) + 1] * 2)
        st = Step(LENGTHS, NEW, dtype=BF16, cache=E4M3, scale=size)
        check(ctx, st, frequencies(32), True, scales=(0.01, 2.0))


def test_infinities_and_nan_stay_in_their_rows(ctx):
    st = Step(LENGTHS, NEW)
    st.qkv[5, 1, 3], st.qkv[6, 2, 9], st.qkv[7, 5, 0] = math.inf, math.nan, -math.inf
    k = kvx()
    qkv = st.qkv.cuda()
    out = torch.full((st.rows, 4, 64), 7.0, dtype=BF16, device="cuda")
    w = torch.ones(64, dtype=BF16, device="cuda")
    k.kv_append_rotary(ctx, st.pool, 0, st.batch, k.KvRotary(4, frequencies(32).cuda(), q_weight=w, k_weight=w), qkv[:, :4], qkv[:, 4:6],
                       qkv[:, 6:], out, starts=ints(st.starts))
    bad = ~torch.isfinite(out).all(-1)
    assert bad.nonzero().tolist() == [[5, 1], [6, 2]]
    st.pages.data = st.dev.cpu()[None]
    for row, s, p in st.owner():
        rows = st.pages.rows(0, st.tables[s], [p])[:, 0]
        odd = ~torch.isfinite(rows.float()).all(-1)
        assert odd.tolist() == [[False, row == 7], [False, False]]


def test_frequencies_that_are_not_finite_or_reach_around_many_times(ctx):
    """Pairs of a frequency that is no number are none; the others are as without it.  Angles of whole turns' many, at places of up to
    2^31, against whole-number arithmetic: within (1 + f) 2^-33 turns and what 32 bits leave of a turn and of its sine, 2^-21 in all."""
    k = kvx()
    pi = 31415926535897932384626433832795028841971693993751058209749445923  # over 10^64
    freq = torch.tensor([1.0, math.nan, 100.0, math.inf, 3e-7, -math.inf, 0.7, 977.25], dtype=torch.float32)
    places = [0, 1, 2 ** 20 + 1, 2 ** 31 - 1]
    st = Step([4], [4], dim=16, dtype=FP16)
    st.qkv[:, :4, :8], st.qkv[:, :4, 8:] = 1.0, 0.0  # rows that become cosines and sines
    out = torch.zeros((4, 4, 16), dtype=FP16, device="cuda")
    qkv = st.qkv.cuda()
    k.kv_append_rotary(ctx, st.pool, 0, st.batch, k.KvRotary(4, freq.cuda()), qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], out, positions=ints(places),
                       new_tokens=4)
    got = out.cpu().double()
    for i, f in enumerate(freq.tolist()):
        for t, place in enumerate(places):
            pair = got[t, 0, [i, i + 8]]
            if not math.isfinite(f):
                assert bool(torch.isnan(pair).all()), (i, t)
                continue
            over, under = f.as_integer_ratio()
            top, bottom = over * place * 10 ** 64, under * 2 * pi  # turns
            angle = 2 * math.pi * ((top % bottom) / bottom)
            off = 2 * math.pi * (1 + f) * 2.0 ** -33 + 2.0 ** -21
            for have, want in zip(pair.tolist(), (math.cos(angle), math.sin(angle))):
                assert abs(have - want) <= off + 2.0 ** -11 * abs(want) + 2.0 ** -25, (f, place)


def test_missing_pages_are_left_out_and_reported(ctx):
    k = kvx()
    st = Step([40, 20], [30, 4])
    st.batch.block_tables[0, 1] = 10 ** 6
    check(ctx, st, frequencies(32), missing={(0, 1)})
    assert k.kv_get_device_error(ctx) == 1
    st = Step([40, 20], [30, 4])
    st.batch._c.max_length = 35  # the first one counts as 35, and its new rows as those up to that
    st.lengths[0] = 35
    check(ctx, st, frequencies(32), missing={(9, 9)})
    assert k.kv_get_device_error(ctx) == st.tables.shape[1]


def test_captured_call_follows_lengths_and_tables(ctx):
    k = kvx()
    st = Step([40, 3], [1, 1])
    qkv, out = st.qkv.cuda(), torch.zeros((2, 4, 64), dtype=BF16, device="cuda")
    rotary = k.KvRotary(4, frequencies(32).cuda())

    def call():
        k.kv_append_rotary(ctx, st.pool, 0, st.batch, rotary, qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], out)

    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        call()
    st.lengths = [39, 2]
    st.batch.lengths.copy_(ints(st.lengths))
    qkv.copy_(normal(qkv.shape, BF16, 77))
    g.replay()
    torch.cuda.synchronize()
    again, pages = out.clone(), st.dev.clone()
    out.zero_()
    call()
    torch.cuda.synchronize()
    assert torch.equal(out, again) and torch.equal(st.dev, pages) and float(again.abs().sum()) > 0


def test_pages_past_four_gib(ctx):
    k = kvx()
    blocks = (5 << 30) // (2 * 16 * 128 * 2)
    layer = torch.zeros((blocks, 2, 1, 16, 128), dtype=BF16, device="cuda")
    pool = k.KvPool.from_tensors([layer], 1, 16)
    batch = k.KvBatch(ints([[0, blocks - 1]]), ints([20]))
    qkv = normal((8, 3, 128), BF16, 5).cuda()
    out = torch.empty((8, 1, 128), dtype=BF16, device="cuda")
    k.kv_append_rotary(ctx, pool, 0, batch, k.KvRotary(1), qkv[:, :1], qkv[:, 1:2], qkv[:, 2:], out, new_tokens=8)
    assert torch.equal(out, qkv[:, :1]) and torch.equal(layer[-1, :, 0, :4], qkv[4:, 1:].transpose(0, 1))


def test_refusals(ctx):
    """Each returns its status before anything is enqueued and leaves the outputs alone."""
    k = kvx()
    st = Step([20, 3], [1, 1])
    qkv = st.qkv.cuda()
    q, key, value = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    out, freq = torch.full((2, 4, 64), 7.0, dtype=BF16, device="cuda"), frequencies(32).cuda()
    plain = k.KvRotary(4, freq)

    def call(status, rotary=plain, q=q, key=key, value=value, out=out, layer=0, **kw):
        with pytest.raises(k.KvxError) as e:
            k.kv_append_rotary(ctx, st.pool, layer, st.batch, rotary, q, key, value, out, **kw)
        assert e.value.status == status, e.value

    call(k.KVX_ERANGE, layer=1)
    call(k.KVX_EINVAL, rotary=k.KvRotary(4, torch.ones(33, device="cuda")))
    call(k.KVX_EINVAL, rotary=k.KvRotary(0, freq), q=q[:, :0], out=out[:, :0])
    call(k.KVX_EINVAL, rotary=k.KvRotary(4, freq, scale=math.inf))
    call(k.KVX_EINVAL, rotary=k.KvRotary(4, freq, eps=-1.0))
    call(k.KVX_EINVAL, rotary=k.KvRotary(4, freq, weight_offset=math.nan))
    call(k.KVX_EINVAL, q=q.half(), key=key.half(), value=value.half(), out=out.half())  # a bf16 cache
    call(k.KVX_EINVAL, k_scale=-1.0)
    call(k.KVX_EINVAL, v_scale=1e-40)
    call(k.KVX_EINVAL, out=torch.zeros((1, 4, 64), dtype=BF16, device="cuda").expand(2, 4, 64))
    call(k.KVX_EALIGN, q=torch.zeros((2, 4, 72), dtype=BF16, device="cuda")[..., 4:68])
    call(k.KVX_EALIGN, rotary=k.KvRotary(4, freq, q_weight=torch.zeros(72, dtype=BF16, device="cuda")[4:68]))
    call(k.KVX_EDEVICE, q=q.cpu())
    call(k.KVX_EDEVICE, out=out.cpu())
    call(k.KVX_EDEVICE, rotary=k.KvRotary(4, freq.cpu()))
    call(k.KVX_EDEVICE, rotary=k.KvRotary(4, freq, k_weight=torch.ones(64, dtype=BF16)))
    call(k.KVX_EDEVICE, positions=torch.zeros(2, dtype=torch.int32))
    other = torch.as_strided(qkv, (2, 4, 64), (64, 128, 1))  # q's memory, other strides
    call(k.KVX_EINVAL, out=other)
    for bad in ({"q": q[:1]}, {"out": out[:, :3]}, {"key": key[:, :1]}, {"positions": ints([1])}, {"starts": ints([0, 1])}):
        args = {"q": q, "key": key, "value": value, "out": out, **{n: v for n, v in bad.items() if n in ("q", "out", "key")}}
        rest = {n: v for n, v in bad.items() if n not in args}
        with pytest.raises(ValueError):
            k.kv_append_rotary(ctx, st.pool, 0, st.batch, plain, args["q"], args["key"], args["value"], args["out"], **rest)
    with pytest.raises(TypeError):
        k.kv_append_rotary(ctx, st.pool, 0, st.batch, plain, q, key, value, out.half())
    with pytest.raises(TypeError):
        k.kv_append_rotary(ctx, st.pool, 0, st.batch, k.KvRotary(4, freq, q_weight=torch.ones(64, device="cuda")), q, key, value, out)
    k.kv_fault_inject("launch")
    call(k.KVX_ECUDA)
    assert bool((out == 7.0).all()) and torch.equal(st.dev.cpu(), st.pages.data[0])
    assert k.kv_get_device_error(ctx) == -1


def test_nothing_to_do(ctx):
    k = kvx()
    st = Step([3], [1])
    empty = k.KvBatch(torch.zeros((0, 4), dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"))
    q = torch.zeros((0, 4, 64), dtype=BF16, device="cuda")
    before = k.kv_ctx_stats(ctx)["kernel_launches"]
    k.kv_append_rotary(ctx, st.pool, 0, empty, k.KvRotary(4), q, q[:, :2], q[:, 2:], q)
    assert k.kv_ctx_stats(ctx)["kernel_launches"] == before
