"""kv_evict against a sort of (weight, position) on the CPU: chosen positions, moved rows, weights and lengths."""
import math

import pytest
import torch

import operator_refs as refs
from gpu_util import kvx

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    k = kvx()
    c = k.kv_ctx_create(0)
    yield c
    k.kv_ctx_destroy(c)


def bits(t):
    return t.cpu().contiguous().view(torch.uint8)


def make(lengths, budget, layers=2, heads=2, block=16, dim=64, dtype=torch.bfloat16, nhd=False, pack=1, seed=1):
    k = kvx()
    fresh = [min(n, budget) for n in lengths]
    tables, blocks = refs.tables_for(list(lengths) + fresh, block * pack, seed, spare=2)
    pages = refs.Pages(layers, blocks, heads, block, dim, dtype, nhd, pack, seed)
    dev = [x.cuda() for x in pages.data]
    pool = k.KvPool.from_tensors(dev, heads, block, k.KVX_LAYOUT_NHD if nhd else k.KVX_LAYOUT_HND, pack)
    return pages, dev, pool, tables[:len(lengths)], tables[len(lengths):]


def check(ctx, lengths, budget, sinks=0, recent=0, weights=None, stream=None, **shape):
    k = kvx()
    pages, dev, pool, old, new = make(lengths, budget, **shape)
    layers, s, h, n = len(dev), len(lengths), pages.heads, max(lengths)
    if weights is None:
        weights = torch.randn((layers, s, h, n + 5), generator=torch.Generator().manual_seed(3)).exp()
    batch = k.KvBatch(old.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), max_length=n)
    kept = torch.full((layers, s, h, budget), 77, dtype=torch.int32, device="cuda")
    new_lengths = torch.full((s,), 77, dtype=torch.int32, device="cuda")
    new_weights = torch.full((layers, s, h, budget), 77.0, device="cuda")
    w_dev, t_dev = weights.cuda(), new.cuda()
    torch.cuda.synchronize()
    k.kv_evict(ctx, pool, batch, w_dev, budget, t_dev, kept, new_lengths, new_weights, sinks=sinks, recent=recent,
               stream=stream)
    torch.cuda.synchronize()
    assert new_lengths.tolist() == [min(x, budget) for x in lengths]
    for l in range(layers):
        for q in range(s):
            for i in range(h):
                want = refs.select(weights[l, q, i].tolist(), lengths[q], budget, sinks, recent)
                m = len(want)
                got = kept[l, q, i].cpu().tolist()
                assert got == want + [-1] * (budget - m), (l, q, i)
                assert torch.equal(bits(new_weights[l, q, i, :m]), bits(weights[l, q, i, want])), (l, q, i)
                assert bool((new_weights[l, q, i, m:] == 77.0).all())
    # the whole pool: fresh pages hold the kept rows, everything else is as it was
    want = refs.Pages(layers, pages.data.shape[1] // pages.pack, h, pages.block, pages.dim, pages.dtype, pages.nhd, pages.pack)
    want.data = pages.data.clone()
    for l in range(layers):
        for q in range(s):
            for i in range(h):
                for to, at in enumerate(kept[l, q, i].tolist()):
                    if at < 0:
                        break
                    row = pages.rows(l, old[q], [at])[:, 0]
                    there = want.rows(l, new[q], [to])[:, 0].clone()
                    there[:, i] = row[:, i]
                    want.put(l, new[q], to, there)
    for l in range(layers):
        assert torch.equal(bits(dev[l]), bits(want.data[l]))
    assert k.kv_get_device_error(ctx) == -1
    return kept


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("nhd", [False, True])
@pytest.mark.parametrize("block,pack,dim", [(16, 1, 64), (3, 2, 96), (32, 1, 256)])
def test_layouts(ctx, dtype, nhd, block, pack, dim):
    check(ctx, [100, 1, 37, 64], 20, sinks=2, recent=5, dtype=dtype, nhd=nhd, block=block, pack=pack, dim=dim)


@pytest.mark.parametrize("length,budget,sinks,recent", [
    (1, 1, 0, 0), (5, 9, 3, 4), (9, 9, 4, 5), (10, 9, 4, 5), (10, 9, 9, 0), (10, 9, 0, 9), (600, 1, 0, 0), (600, 1, 1, 0),
    (600, 1, 0, 1), (513, 512, 0, 0), (2049, 300, 4, 64), (4096, 1024, 4, 128), (4097, 4096, 0, 1), (0, 3, 1, 1)])
def test_lengths_and_budgets(ctx, length, budget, sinks, recent):
    check(ctx, [length, max(1, length // 2)], budget, sinks, recent, layers=1, heads=1, dim=16)


@pytest.mark.parametrize("kind", ["equal", "two values", "zeros of both signs", "odd values", "denormals", "negative", "nearly equal"])
def test_ties_and_odd_weights(ctx, kind):
    g = torch.Generator().manual_seed(5)
    n = 1500
    if kind == "equal":
        w = torch.full((1, 1, 2, n), 0.5)
    elif kind == "two values":
        w = (torch.rand((1, 1, 2, n), generator=g) > 0.6).float()
    elif kind == "zeros of both signs":
        w = torch.where(torch.rand((1, 1, 2, n), generator=g) > 0.5, 0.0, -0.0)
    elif kind == "odd values":
        w = torch.randn((1, 1, 2, n), generator=g)
        pick = torch.rand(w.shape, generator=g)
        w[pick > 0.7] = math.nan
        w[(pick > 0.5) & (pick <= 0.7)] = -math.inf
        w[pick < 0.1] = math.inf
    elif kind == "denormals":
        w = torch.randint(0, 50, (1, 1, 2, n), generator=g).float() * 1e-45
    elif kind == "negative":
        w = -torch.rand((1, 1, 2, n), generator=g)
    else:
        w = 1.0 + torch.randint(0, 3, (1, 1, 2, n), generator=g).float() * 2.0 ** -23
    for budget in (7, 400, 1100):
        check(ctx, [n], budget, sinks=1, recent=2, weights=w, layers=1, heads=2, dim=16)


def test_nothing_but_nan_still_keeps_the_first(ctx):
    kept = check(ctx, [300], 10, sinks=0, recent=0, weights=torch.full((1, 1, 1, 300), math.nan), layers=1, heads=1, dim=16)
    assert kept[0, 0, 0].tolist() == list(range(10))


def test_long_rows(ctx):
    """Rows of a hundred thousand weights, a few values in many places among them."""
    k = kvx()
    n, budget = 100003, 5000
    g = torch.Generator().manual_seed(6)
    w = torch.randn((1, 2, 1, n), generator=g).exp()
    w[0, 1] = torch.randint(0, 40, (1, n), generator=g).float() * 1e-3
    lengths = [n, n - 77]
    tables, blocks = refs.tables_for(lengths + [budget, budget], 64, 6)
    layer = torch.randint(0, 255, (blocks, 2, 1, 64, 16), dtype=torch.uint8, generator=g).cuda()
    pool = k.KvPool.from_tensors([layer], 1, 64)
    batch = k.KvBatch(tables[:2].cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), max_length=n)
    kept = torch.zeros((1, 2, 1, budget), dtype=torch.int32, device="cuda")
    new_lengths = torch.zeros(2, dtype=torch.int32, device="cuda")
    k.kv_evict(ctx, pool, batch, w.cuda(), budget, tables[2:].cuda(), kept, new_lengths, sinks=4, recent=100)
    torch.cuda.synchronize()
    data = layer.cpu()
    for s in range(2):
        want = refs.select(w[0, s, 0].tolist(), lengths[s], budget, 4, 100)
        assert kept[0, s, 0].tolist() == want
        at, to = torch.tensor(want), torch.arange(budget)
        assert torch.equal(data[tables[s][at // 64].long(), :, 0, at % 64], data[tables[2 + s][to // 64].long(), :, 0, to % 64])


@pytest.mark.parametrize("width", [0, 1])  # rows of weights on 16 bytes, and off them
@pytest.mark.parametrize("n", [4096, 12288, 12289, 32768, 32769])
def test_rows_that_just_fill_a_tile(ctx, n, width):
    k = kvx()
    budget = 700
    w = torch.randn((1, 1, 2, (n + 3) // 4 * 4 + width), generator=torch.Generator().manual_seed(8)).exp()
    w[0, 0, 1] = torch.randint(0, 30, (w.shape[-1],), generator=torch.Generator().manual_seed(9)).float()
    tables, blocks = refs.tables_for([n, budget], 64, 6)
    layer = torch.zeros((blocks, 2, 2, 64, 16), dtype=torch.uint8, device="cuda")
    pool = k.KvPool.from_tensors([layer], 2, 64)
    batch = k.KvBatch(tables[:1].cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"), max_length=n)
    kept = torch.zeros((1, 1, 2, budget), dtype=torch.int32, device="cuda")
    new_lengths = torch.zeros(1, dtype=torch.int32, device="cuda")
    k.kv_evict(ctx, pool, batch, w.cuda(), budget, tables[1:].cuda(), kept, new_lengths, sinks=3, recent=5)
    for h in range(2):
        assert kept[0, 0, h].tolist() == refs.select(w[0, 0, h].tolist(), n, budget, 3, 5)


def test_on_another_stream_after_the_attention_that_weighs(ctx):
    """Attention on a side stream accumulates the weights that the eviction behind it on that stream reads."""
    k = kvx()
    n, budget = 400, 60
    pages, dev, pool, old, new = make([n], budget, layers=1, heads=1, dim=64)
    batch = k.KvBatch(old.cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"))
    att = k.KvAttention(4)
    longest = old.shape[1] * 16
    weights = torch.zeros((1, 1, 1, longest), device="cuda")
    ws = k.kv_attend_workspace(ctx, pool, batch, att, weights=True)
    q = torch.randn((1, 4, 64), generator=torch.Generator().manual_seed(7)).to(torch.bfloat16).cuda()
    out = torch.empty_like(q)
    kept = torch.zeros((1, 1, 1, budget), dtype=torch.int32, device="cuda")
    new_lengths = torch.zeros(1, dtype=torch.int32, device="cuda")
    t_dev = new.cuda()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        k.kv_attend(ctx, pool, 0, batch, att, q, out, ws, weights=weights[0])
        k.kv_evict(ctx, pool, batch, weights, budget, t_dev, kept, new_lengths, sinks=1, recent=8)
    side.synchronize()
    assert abs(float(weights.sum()) - 4.0) < 1e-4
    assert kept[0, 0, 0].tolist() == refs.select(weights[0, 0, 0].tolist(), n, budget, 1, 8)


def test_missing_pages(ctx):
    """A kept token whose old page is missing leaves zeros, one without a new page is not written; both are reported."""
    k = kvx()
    pages, dev, pool, old, new = make([40], 20, layers=1, heads=1)
    old[0, 0] = -1
    new[0, 1] = 10 ** 6
    before = dev[0].clone()
    batch = k.KvBatch(old.cuda(), torch.tensor([40], dtype=torch.int32, device="cuda"), max_length=48)
    w = torch.arange(48, 0, -1, dtype=torch.float32, device="cuda").view(1, 1, 1, 48)
    kept = torch.zeros((1, 1, 1, 20), dtype=torch.int32, device="cuda")
    new_lengths = torch.zeros(1, dtype=torch.int32, device="cuda")
    k.kv_evict(ctx, pool, batch, w, 20, new.cuda(), kept, new_lengths)
    torch.cuda.synchronize()
    assert kept[0, 0, 0].tolist() == list(range(20))
    assert k.kv_get_device_error(ctx) == 0
    before[int(new[0, 0])] = 0
    assert torch.equal(bits(dev[0]), bits(before))


@pytest.mark.parametrize("stride", [2 ** 60, 2 ** 61, 2 ** 62, 2 ** 63 - 1])
@pytest.mark.parametrize("which", ["block_tables", "new_tables"])
def test_table_strides_beyond_64_bits_of_bytes(ctx, stride, which):
    """Their products with the sequences must not wrap into a small extent."""
    import ctypes
    k = kvx()
    lengths = [40, 9, 1, 3, 20]
    pages, dev, pool, old, new = make(lengths, 8)
    batch = k.KvBatch(old.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), max_length=40)
    w, t = torch.zeros((2, 5, 2, 40), device="cuda"), new.cuda()
    kept, out = torch.full((2, 5, 2, 8), 77, dtype=torch.int32, device="cuda"), torch.full((5,), 77, dtype=torch.int32, device="cuda")
    e = k.kvx_eviction(8, 0, 0, w.data_ptr(), *w.stride()[:3], t.data_ptr(), t.stride(0), t.shape[1], kept.data_ptr(), out.data_ptr())
    if which == "block_tables":
        batch._c.table_stride = stride
    else:
        e.new_table_stride = stride
    status = k._lib.kv_evict(ctx, ctypes.byref(pool._c), ctypes.byref(batch._c), ctypes.byref(e), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert status == k.KVX_EINVAL
    assert bool((kept == 77).all()) and bool((out == 77).all())


@pytest.mark.parametrize("dim", [0, 1, 2])
def test_new_weights_that_lie_over_one_another(ctx, dim):
    """Layers, sequences or heads that share their rows of new weights would be written over one another."""
    k = kvx()
    pages, dev, pool, old, new = make([40, 9], 8)
    batch = k.KvBatch(old.cuda(), torch.tensor([40, 9], dtype=torch.int32, device="cuda"), max_length=40)
    w = torch.zeros((2, 2, 2, 40), device="cuda")
    kept, out = torch.full((2, 2, 2, 8), 77, dtype=torch.int32, device="cuda"), torch.full((2,), 77, dtype=torch.int32, device="cuda")
    shape = [2, 2, 2, 8]
    shape[dim] = 1
    shared = torch.full(shape, 77.0, device="cuda").expand(2, 2, 2, 8)
    with pytest.raises(k.KvxError) as e:
        k.kv_evict(ctx, pool, batch, w, 8, new.cuda(), kept, out, shared)
    assert e.value.status == k.KVX_EINVAL
    torch.cuda.synchronize()
    assert bool((kept == 77).all()) and bool((out == 77).all()) and bool((shared == 77.0).all())
    # rows in another order are not shared
    k.kv_evict(ctx, pool, batch, w, 8, new.cuda(), kept, out, torch.zeros((2, 2, 2, 8), device="cuda").permute(2, 0, 1, 3))
    torch.cuda.synchronize()
    assert out.tolist() == [8, 8]


def test_refusals(ctx):
    k = kvx()
    pages, dev, pool, old, new = make([40, 9], 8)
    lengths = torch.tensor([40, 9], dtype=torch.int32, device="cuda")
    batch = k.KvBatch(old.cuda(), lengths, max_length=40)
    w = torch.zeros((2, 2, 2, 40), device="cuda")
    kept = torch.full((2, 2, 2, 8), 77, dtype=torch.int32, device="cuda")
    out = torch.full((2,), 77, dtype=torch.int32, device="cuda")
    t = new.cuda()

    def refuse(status, budget=8, tables=t, kept=kept, out=out, batch=batch, w=w, **kw):
        with pytest.raises(k.KvxError) as e:
            k.kv_evict(ctx, pool, batch, w, budget, tables, kept, out, **kw)
        assert e.value.status == status, e.value

    refuse(k.KVX_EINVAL, sinks=5, recent=4)
    refuse(k.KVX_EINVAL, sinks=-1)
    refuse(k.KVX_EINVAL, budget=0, kept=kept[..., :0].contiguous())
    refuse(k.KVX_ERANGE, budget=17, tables=t[:, :1], kept=torch.zeros((2, 2, 2, 17), dtype=torch.int32, device="cuda"))
    refuse(k.KVX_EINVAL, out=lengths)
    refuse(k.KVX_EDEVICE, w=w.cpu())
    with pytest.raises(ValueError):
        k.kv_evict(ctx, pool, batch, w[..., :39], 8, t, kept, out)
    with pytest.raises(TypeError):
        k.kv_evict(ctx, pool, batch, w, 8, t, kept.long(), out)
    assert bool((kept == 77).all()) and bool((out == 77).all())
    for d, p in zip(dev, pages.data):
        assert torch.equal(bits(d), bits(p))
