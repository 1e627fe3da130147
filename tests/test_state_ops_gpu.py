"""kv_state_conv and kv_state_scan against token-by-token 64-bit recurrences."""
import math

import pytest
import torch

import operator_refs as refs
from gpu_util import kvx

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16


def normal(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


@pytest.fixture(scope="module")
def ctx():
    k = kvx()
    c = k.kv_ctx_create(0)
    yield c
    k.kv_ctx_destroy(c)


class Slots:
    """Slots of a recurrent state and a window each, all of random numbers, on the CPU and the GPU."""

    def __init__(self, n, heads=1, p=8, state=16, width=4, channels=8, dtype=BF16, seed=1):
        k = kvx()
        self.rec, self.win = heads * p * state * 4, (width - 1) * channels * 2
        self.bytes = -(-(self.rec + self.win) // 256) * 256 + 256
        self.n, self.dtype = n, dtype
        self.cpu = torch.zeros((n, self.bytes), dtype=torch.uint8)
        self.state = self.cpu[:, :self.rec].view(torch.float32).view(n, heads, p, state)
        self.window = self.cpu[:, self.rec:self.rec + self.win].view(dtype).view(n, width - 1, channels)
        self.state.copy_(normal(self.state.shape, torch.float32, seed))
        self.window.copy_(normal(self.window.shape, dtype, seed + 1))
        self.cpu[:, self.rec + self.win:] = 0xA5  # padding that nothing may touch
        self.dev = self.cpu.cuda()
        self.slots = k.StateSlots(self.dev, n, self.bytes, recurrent_offset=0, conv_offset=self.rec)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def batch_of(lens, slots_in, slots_out=None, fresh=None, single=False):
    k = kvx()
    starts = [sum(lens[:i]) for i in range(len(lens) + 1)]
    return k.StateBatch(ints(slots_in), None if slots_out is None else ints(slots_out),
                        starts=None if single else ints(starts), tokens=starts[-1],
                        fresh=None if fresh is None else ints(fresh)), starts


def check_conv(ctx, lens, channels, width, dtype, bias=True, silu=True, single=False, in_place=False, fresh=None, stream=None):
    k = kvx()
    s = len(lens)
    st = Slots(2 * s + 1, width=width, channels=channels, dtype=dtype)
    ins = [(3 * i + 1) % (2 * s + 1) for i in range(s)] if in_place else list(range(s, 0, -1))
    outs = ins if in_place else [s + 1 + i for i in range(s)]
    if in_place and len(set(ins)) < s:
        ins = outs = list(range(s))
    batch, starts = batch_of(lens, ins, None if in_place else outs, fresh, single)
    t = starts[-1]
    wide = normal((t, channels + 24), dtype, 3)
    x, w = wide[:, 8:8 + channels], normal((channels, width), dtype, 4, 0.6)
    b = normal((channels,), dtype, 5) if bias else None
    out = torch.full((t, channels + 8), 7.0, dtype=dtype, device="cuda")
    dev = wide.cuda()
    w_dev, b_dev = w.cuda(), None if b is None else b.cuda()
    torch.cuda.synchronize()
    k.kv_state_conv(ctx, st.slots, batch, dev[:, 8:8 + channels], w_dev, out[:, :channels], bias=b_dev, silu=silu, stream=stream)
    torch.cuda.synchronize()
    unit = refs.UNIT[dtype]
    want = st.cpu.clone()
    windows = want[:, st.rec:st.rec + st.win].view(dtype).view(st.n, width - 1, channels)
    for i in range(s):
        first = torch.zeros_like(st.window[0]).double() if fresh and fresh[i] else st.window[ins[i]].double()
        rows = x[starts[i]:starts[i + 1]].double()
        y, window = refs.conv(rows, w.double(), None if b is None else b.double(), first, silu)
        size, _ = refs.conv(rows.abs(), w.double().abs(), None if b is None else b.double().abs(), first.abs(), False)
        # a sum of width products and a bias in 32 bits, and y * sigmoid(y), whose slope is below 1.1; then one rounding
        bound = unit * y.abs() + 2.0 ** -20 * size + 1e-7
        got = out[starts[i]:starts[i + 1], :channels].cpu().double()
        assert bool(((got - y).abs() <= bound).all()), i
        windows[outs[i]] = window.to(dtype)
    assert bool((out[:, channels:] == 7.0).all())
    assert torch.equal(st.dev.cpu(), want)
    assert k.kv_get_device_error(ctx) == -1


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("width", [2, 3, 4])
@pytest.mark.parametrize("in_place", [False, True])
def test_conv_prompts(ctx, dtype, width, in_place):
    check_conv(ctx, [0, 1, 2, 3, 70, 129, 600], 72, width, dtype, in_place=in_place)


@pytest.mark.parametrize("channels", [8, 264, 2048, 8192])
@pytest.mark.parametrize("seqs", [1, 5])
def test_conv_single_tokens(ctx, channels, seqs):
    check_conv(ctx, [1] * seqs, channels, 4, BF16, single=True)
    check_conv(ctx, [1] * seqs, channels, 3, FP16, single=True, in_place=True, bias=False)


@pytest.mark.parametrize("silu,bias", [(True, False), (False, True), (False, False)])
def test_conv_options_and_fresh_sequences(ctx, silu, bias):
    check_conv(ctx, [2, 5, 1, 40], 40, 4, BF16, silu=silu, bias=bias, fresh=[0, 1, 1, 0], stream=torch.cuda.Stream())


def scan_inputs(t, heads, p, n, groups, dtype, seed=3, fast=False):
    """fast: decays from none at all to one that forgets within a token."""
    wide = normal((t, heads * p + 2 * groups * n + 8), dtype, seed)
    x = wide[:, :heads * p].view(t, heads, p)
    b = wide[:, heads * p:heads * p + groups * n].view(t, groups, n)
    c = wide[:, heads * p + groups * n:heads * p + 2 * groups * n].view(t, groups, n)
    g = torch.Generator().manual_seed(seed + 1)
    dt = normal((t, heads), dtype, seed + 2, 3.0 if fast else 1.0)
    A = -torch.exp(torch.rand(heads, generator=g) * (8.0 if fast else 2.5) - (5.0 if fast else 0.0))
    return wide, x, b, c, dt, A, torch.randn(heads, generator=g), torch.randn(heads, generator=g) - 4.0


def check_scan(ctx, lens, heads, p, n, groups, dtype, single=False, in_place=False, fresh=None, softplus=True, skip=True,
               bias=True, fast=False, stream=None):
    k = kvx()
    s = len(lens)
    st = Slots(2 * s + 1, heads, p, n, dtype=dtype)
    ins = list(range(s)) if in_place else list(range(s, 0, -1))
    outs = ins if in_place else [s + 1 + i for i in range(s)]
    batch, starts = batch_of(lens, ins, None if in_place else outs, fresh, single)
    t = starts[-1]
    wide, x, b, c, dt, A, D, dt_bias = scan_inputs(t, heads, p, n, groups, dtype, fast=fast)
    if not softplus:
        dt = (dt.abs() * 0.02).to(dtype)
    dev = wide.cuda()
    dx = dev[:, :heads * p].view(t, heads, p)
    db = dev[:, heads * p:heads * p + groups * n].view(t, groups, n)
    dc = dev[:, heads * p + groups * n:heads * p + 2 * groups * n].view(t, groups, n)
    out = torch.full((t, heads * p + 8), 7.0, dtype=dtype, device="cuda")
    use_bias = bias and softplus
    ws = k.kv_state_scan_workspace(ctx, batch, heads, p, n)
    ws.fill_(0xFF)  # NaN: nothing of it may be read before it is written
    args = dt.cuda(), A.cuda(), D.cuda() if skip else None, dt_bias.cuda() if use_bias else None
    torch.cuda.synchronize()
    k.kv_state_scan(ctx, st.slots, batch, dx, args[0], args[1], db, dc, out[:, :heads * p].view(t, heads, p), D=args[2],
                    dt_bias=args[3], softplus=softplus, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    unit = refs.UNIT[dtype]
    got_state = st.dev.cpu()[:, :st.rec].view(torch.float32).view(st.state.shape)
    untouched = st.cpu.clone()
    for i in range(s):
        rows = slice(starts[i], starts[i + 1])
        first = torch.zeros_like(st.state[0]).double() if fresh and fresh[i] else st.state[ins[i]].double()
        y, state, size, big = refs.scan(x[rows].double(), dt[rows].double(), A.double(), b[rows].double(), c[rows].double(),
                                        D.double() if skip else None, dt_bias.double() if use_bias else None, softplus, first)
        # Products of matrices round up to three factors of a term to the inputs' type (a pair's decayed product, a
        # decayed input, a carried state); the rest is in 32 bits, with decays from exponents of up to some hundreds.
        got = out[rows, :heads * p].view(-1, heads, p).cpu().double()
        bound = unit * y.abs() + (3 * unit + 2.0 ** -13) * size + 1e-7
        assert bool(((got - y).abs() <= bound).all()), (i, float(((got - y).abs() / bound).max()))
        off = (got_state[outs[i]].double() - state).abs()
        assert bool((off <= 2.0 ** -14 * big + 1e-9).all()), (i, float((off / (big + 1e-9)).max()))
        untouched[outs[i], :st.rec] = st.dev.cpu()[outs[i], :st.rec]
    assert bool((out[:, heads * p:] == 7.0).all())
    assert torch.equal(st.dev.cpu(), untouched)
    assert k.kv_get_device_error(ctx) == -1


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("p", [8, 64, 120, 128, 256])
@pytest.mark.parametrize("n", [16, 32, 64, 128, 256])
def test_scan_single_tokens(ctx, dtype, p, n):
    check_scan(ctx, [1, 1, 1], 4, p, n, 2, dtype, single=True, in_place=n == 64)


# lengths around the 64 and 128 tokens of a chunk, of one token and of none
LENS = [0, 1, 2, 63, 64, 65, 127, 128, 129, 300]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("p,n,heads,groups", [(64, 64, 2, 1), (64, 128, 4, 2), (128, 64, 3, 3), (128, 128, 2, 1)])
def test_scan_prompts(ctx, dtype, p, n, heads, groups):
    check_scan(ctx, LENS, heads, p, n, groups, dtype)
    check_scan(ctx, [200, 5], heads, p, n, groups, dtype, in_place=True, fresh=[1, 0])


@pytest.mark.parametrize("p,n", [(8, 16), (40, 32), (256, 64), (64, 256), (72, 128), (16, 16)])
def test_scan_prompts_of_other_sizes(ctx, p, n):
    check_scan(ctx, [0, 1, 40, 150], 2, p, n, 1, BF16)


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_scan_of_short_and_long_sequences_together(ctx, dtype):
    """Around the 16 tokens up to which a sequence of a batch goes token by token, with more sequences than a warp has lanes."""
    check_scan(ctx, [17, 16, 15, 0, 400, 1], 2, 128, 128, 1, dtype, fresh=[0, 1, 0, 0, 1, 0])
    check_scan(ctx, [17, 0, 1, 16, 3, 1, 2, 2], 2, 128, 128, 1, dtype, fresh=[0, 1, 0, 0, 1, 0, 0, 0])
    check_scan(ctx, [17, 16, 15, 0, 400, 1], 52, 128, 128, 4, dtype)
    check_scan(ctx, [3, 16, 17, 0, 2] * 7 + [200, 1, 90], 2, 64, 64, 2, dtype, in_place=True)
    check_scan(ctx, [16, 16, 16], 2, 128, 64, 1, dtype)


@pytest.mark.parametrize("t", [1, 16, 17, 384, 385, 520])
def test_scan_of_one_sequence(ctx, t):
    check_scan(ctx, [t], 3, 128, 128, 1, BF16)


def test_scan_long_prompt(ctx):
    check_scan(ctx, [1500, 700], 2, 128, 128, 1, BF16)


@pytest.mark.parametrize("softplus,skip,bias", [(False, True, False), (True, False, True), (True, True, False), (False, False, False)])
def test_scan_options(ctx, softplus, skip, bias):
    check_scan(ctx, [150, 1, 30], 2, 64, 128, 1, BF16, softplus=softplus, skip=skip, bias=bias, stream=torch.cuda.Stream())


def test_scan_of_fast_and_slow_decays(ctx):
    """Heads that forget within a token beside heads that forget nothing: exponents of thousands over a chunk."""
    check_scan(ctx, [260, 70], 8, 64, 64, 1, BF16, fast=True, bias=False)


def test_fresh_sequences_do_not_read_their_slots(ctx):
    """A fresh sequence's slot may hold anything, NaN too."""
    k = kvx()
    for lens, single in (([1, 1], True), ([130, 3], False)):
        st = Slots(2, 2, 64, 64)
        st.dev.fill_(0xFF)
        batch, starts = batch_of(lens, [1, 0], fresh=[1, 1], single=single)
        t = starts[-1]
        wide, x, b, c, dt, A, D, dt_bias = scan_inputs(t, 2, 64, 64, 1, BF16)
        out = torch.empty((t, 2, 64), dtype=BF16, device="cuda")
        k.kv_state_scan(ctx, st.slots, batch, x.cuda(), dt.cuda(), A.cuda(), b.cuda(), c.cuda(), out,
                        workspace=k.kv_state_scan_workspace(ctx, batch, 2, 64, 64))
        cv = torch.empty((t, 8), dtype=BF16, device="cuda")
        k.kv_state_conv(ctx, st.slots, batch, normal((t, 8), BF16, 8).cuda(), normal((8, 4), BF16, 9).cuda(), cv)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(cv).all())
        assert bool(torch.isfinite(st.dev[:, :st.rec].view(torch.float32)).all())


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("p,skip", [(64, True), (128, False), (8, True)])
def test_scan_of_infinities_and_nan(ctx, dtype, p, skip):
    """An input that is not finite reaches its own row of the state from its token on, and nothing before it."""
    k = kvx()
    t, heads, n = 300, 2, 64
    wide, x, b, c, dt, A, D, dt_bias = scan_inputs(t, heads, p, n, 1, dtype)
    x[70, 0, 3], x[150, 1, 5], x[151, 1, 6], x[299, 0, 7] = math.inf, math.nan, -math.inf, math.nan
    st = Slots(1, heads, p, n, dtype=dtype)
    batch, _ = batch_of([t], [0])
    out = torch.empty((t, heads, p), dtype=dtype, device="cuda")
    k.kv_state_scan(ctx, st.slots, batch, x.cuda(), dt.cuda(), A.cuda(), b.cuda(), c.cuda(), out, D=D.cuda() if skip else None,
                    workspace=k.kv_state_scan_workspace(ctx, batch, heads, p, n))
    torch.cuda.synchronize()
    y, state, size, big = refs.scan(x.double(), dt.double(), A.double(), b.double(), c.double(), D.double() if skip else None,
                                    None, True, st.state[0].double())
    got = out.cpu().double()
    fine = torch.isfinite(y)
    assert torch.equal(torch.isfinite(got), fine)
    unit = refs.UNIT[dtype]
    assert bool(((got - y).abs()[fine] <= (unit * y.abs() + (3 * unit + 2.0 ** -13) * size + 1e-7)[fine]).all())
    after = st.dev.cpu()[0, :st.rec].view(torch.float32).view(state.shape).double()
    fine = torch.isfinite(state)
    assert torch.equal(torch.isfinite(after), fine)
    assert bool(((after - state).abs()[fine] <= (2.0 ** -14 * big + 1e-9)[fine]).all())


@pytest.mark.parametrize("bc,size_x,step", [(0.01, 1000.0, 1e-3), (0.03, 100.0, 1e-3), (1.0, 1.0, 2e-6), (1.0, 1.0, 1.0), (64.0, 1e-3, 1.0),
                                            (250.0, 1e-4, 3.0)])
@pytest.mark.parametrize("p,n", [(64, 64), (128, 128)])
def test_scan_of_small_and_large_factors_in_fp16(ctx, bc, size_x, step, p, n):
    """A chunk of small or large B, C and steps, whose decayed products M = (C . B) e^.. d leave the range in which fp16
    has its 11 bits, or fp16's altogether, where the results do not."""
    k = kvx()
    t, heads = 128, 2
    wide, x, b, c, dt, A, D, dt_bias = scan_inputs(t, heads, p, n, 1, FP16, seed=31)
    x, b, c = (x * size_x).to(FP16), (b * bc).to(FP16), (c * bc).to(FP16)
    dt = (torch.rand((t, heads), generator=torch.Generator().manual_seed(32)) * step).to(FP16)
    st = Slots(1, heads, p, n, dtype=FP16)
    batch, _ = batch_of([t], [0], fresh=[1])
    out = torch.empty((t, heads, p), dtype=FP16, device="cuda")
    k.kv_state_scan(ctx, st.slots, batch, x.cuda(), dt.cuda(), A.cuda(), b.cuda(), c.cuda(), out, softplus=False,
                    workspace=k.kv_state_scan_workspace(ctx, batch, heads, p, n))
    torch.cuda.synchronize()
    y, _, size, _ = refs.scan(x.double(), dt.double(), A.double(), b.double(), c.double(), None, None, False,
                              torch.zeros((heads, p, n), dtype=torch.float64))
    assert float(y.abs().max()) < 65504
    exponent = torch.cumsum(dt.double() * A.double(), 0).T  # [head][token]
    decay = torch.exp((exponent[:, :, None] - exponent[:, None, :]).masked_fill(~torch.ones(t, t, dtype=torch.bool).tril(), -math.inf))
    m = (c[:, 0].double() @ b[:, 0].double().T) * decay * dt.double().T[:, None, :]
    rounded = (m.abs() @ x.double().abs().permute(1, 0, 2)).permute(1, 0, 2)  # what one rounding a term is relative to
    # a rounding of M and of y, exponents of some hundreds and C . B in 32 bits; y's own subnormals
    unit = refs.UNIT[FP16]
    bound = unit * y.abs() + (unit + 2.0 ** -13) * rounded + 2.0 ** -19 * size + 2.0 ** -25
    off = (out.cpu().double() - y).abs()
    assert bool((off <= bound).all()), float((off / bound).max())


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("p,n", [(64, 64), (128, 128)])
def test_scan_of_slow_decays_behind_fast_ones(ctx, dtype, p, n):
    """Tokens that forget everything, then tokens that forget little: a decay is taken of the tokens between two, however
    large the exponents before them are."""
    k = kvx()
    t, heads = 128, 4
    wide, x, b, c, dt, A, D, dt_bias = scan_inputs(t, heads, p, n, 1, dtype, seed=33)
    A = -torch.tensor([8.0, 80.0, 800.0, 8e6])  # exponents of 2e3, 2e4, 2e5 and 2e9 before the slow tokens
    slow = torch.tensor([1e-5, 5e-6, 5e-6, 1e-7]) * torch.rand((t, heads), generator=torch.Generator().manual_seed(34))
    dt = torch.where(torch.arange(t)[:, None] < 64, torch.tensor(3.0), slow).to(dtype)
    st = Slots(1, heads, p, n, dtype=dtype)
    batch, _ = batch_of([t], [0], fresh=[1])
    out = torch.empty((t, heads, p), dtype=dtype, device="cuda")
    k.kv_state_scan(ctx, st.slots, batch, x.cuda(), dt.cuda(), A.cuda(), b.cuda(), c.cuda(), out, softplus=False,
                    workspace=k.kv_state_scan_workspace(ctx, batch, heads, p, n))
    torch.cuda.synchronize()
    y, _, size, _ = refs.scan(x.double(), dt.double(), A.double(), b.double(), c.double(), None, None, False,
                              torch.zeros((heads, p, n), dtype=torch.float64))
    exponent = torch.cumsum(dt.double() * A.double(), 0).T  # [head][token]
    decay = torch.exp((exponent[:, :, None] - exponent[:, None, :]).masked_fill(~torch.ones(t, t, dtype=torch.bool).tril(), -math.inf))
    m = (c[:, 0].double() @ b[:, 0].double().T) * decay * dt.double().T[:, None, :]
    rounded = (m.abs() @ x.double().abs().permute(1, 0, 2)).permute(1, 0, 2)
    # a rounding of M and of y; an exponent of up to 30 (beyond which a term is nothing) in 32 bits, and C . B
    unit = refs.UNIT[dtype]
    bound = unit * y.abs() + (unit + 2.0 ** -16) * rounded + 2.0 ** -19 * size + 2.0 ** -25
    off = (out.cpu().double() - y).abs()
    assert bool((off <= bound).all()), float((off / bound).max())


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("p,n", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("t", [40, 128, 300, 520])
def test_state_keeps_the_bits_of_the_weighted_inputs(ctx, dtype, p, n, t):
    """One token a head has an input, so an element of the state is one product, decayed: nothing averages out what a
    split of the weighted input (three bf16 numbers, two of fp16: 24 and 22 bits) would lose."""
    k = kvx()
    heads = 4
    wide, x, b, c, dt, A, D, dt_bias = scan_inputs(t, heads, p, n, 1, dtype, seed=41)
    x = x.clone()
    for h, at in enumerate([3, t // 3, t // 2, t - 1]):
        x[:at, h], x[at + 1:, h] = 0, 0
    dt = torch.full((t, heads), 2.0 ** -10).to(dtype)
    A = -torch.tensor([0.3, 0.5, 0.7, 0.9])
    st = Slots(1, heads, p, n, dtype=dtype)
    batch, _ = batch_of([t], [0], fresh=[1])
    out = torch.empty((t, heads, p), dtype=dtype, device="cuda")
    k.kv_state_scan(ctx, st.slots, batch, x.cuda(), dt.cuda(), A.cuda(), b.cuda(), c.cuda(), out, softplus=False,
                    workspace=k.kv_state_scan_workspace(ctx, batch, heads, p, n))
    torch.cuda.synchronize()
    _, state, _, _ = refs.scan(x.double(), dt.double(), A.double(), b.double(), c.double(), None, None, False,
                               torch.zeros((heads, p, n), dtype=torch.float64))
    got = st.dev.cpu()[0, :st.rec].view(torch.float32).view(heads, p, n).double()
    # 2^-22 of the split, 2^-22 of each of up to five chunks' powers of two, three sums of products in 32 bits
    assert bool(((got - state).abs() <= 2.0 ** -19 * state.abs()).all())


def test_scan_of_fast_and_slow_decays_in_fp16(ctx):
    check_scan(ctx, [260, 70], 8, 64, 64, 1, FP16, fast=True, bias=False)
    check_scan(ctx, [700], 8, 128, 128, 2, FP16, fast=True, bias=False)


def test_token_by_token_is_the_prompt(ctx):
    """A prompt in one call and its tokens one by one leave the same state within the bounds of both."""
    k = kvx()
    t, heads, p, n = 90, 2, 64, 64
    wide, x, b, c, dt, A, D, dt_bias = scan_inputs(t, heads, p, n, 1, BF16)
    dev = [v.cuda() for v in (x, dt, A, b, c)]
    st, one = Slots(1, heads, p, n), Slots(1, heads, p, n)
    out, outs = torch.empty((t, heads, p), dtype=BF16, device="cuda"), torch.empty((t, heads, p), dtype=BF16, device="cuda")
    batch, _ = batch_of([t], [0])
    k.kv_state_scan(ctx, st.slots, batch, dev[0], dev[1], dev[2], dev[3], dev[4], out,
                    workspace=k.kv_state_scan_workspace(ctx, batch, heads, p, n))
    single = k.StateBatch(ints([0]))
    for i in range(t):
        r = slice(i, i + 1)
        k.kv_state_scan(ctx, one.slots, single, dev[0][r], dev[1][r], dev[2], dev[3][r], dev[4][r], outs[r])
    torch.cuda.synchronize()
    _, _, size, big = refs.scan(x.double(), dt.double(), A.double(), b.double(), c.double(), None, None, True, st.state[0].double())
    a = st.dev.cpu()[:, :st.rec].view(torch.float32).double().view(heads, p, n)
    z = one.dev.cpu()[:, :st.rec].view(torch.float32).double().view(heads, p, n)
    assert bool(((a - z).abs() <= 2.0 ** -13 * big + 1e-9).all())
    assert bool(((out.cpu().double() - outs.cpu().double()).abs() <= 5 * refs.UNIT[BF16] * size + 1e-6).all())


def test_bad_slots_give_zeros_and_are_reported(ctx):
    k = kvx()
    for lens, single in (([1, 1, 1], True), ([100, 70, 3], False)):
        st = Slots(3, 2, 64, 64)
        batch, starts = batch_of(lens, [0, 5, 1], [0, 1, -1], single=single)
        t = starts[-1]
        wide, x, b, c, dt, A, D, dt_bias = scan_inputs(t, 2, 64, 64, 1, BF16)
        out = torch.full((t, 2, 64), math.nan, dtype=BF16, device="cuda")
        k.kv_state_scan(ctx, st.slots, batch, x.cuda(), dt.cuda(), A.cuda(), b.cuda(), c.cuda(), out, D=D.cuda(),
                        workspace=k.kv_state_scan_workspace(ctx, batch, 2, 64, 64))
        cv = torch.full((t, 8), 7.0, dtype=BF16, device="cuda")
        k.kv_state_conv(ctx, st.slots, batch, normal((t, 8), BF16, 8).cuda(), normal((8, 4), BF16, 9).cuda(), cv)
        torch.cuda.synchronize()
        assert bool((out[starts[1]:] == 0).all()) and bool((cv[starts[1]:] == 0).all())
        assert bool(torch.isfinite(out[:starts[1]]).all())
        assert torch.equal(st.dev.cpu()[1:], st.cpu[1:])
        assert k.kv_get_device_error(ctx) == 1


@pytest.mark.parametrize("starts", [[0, 3000, 0, 3000], [3000, 0, 3000, 0, 3000], [0, 3000] * 20])
def test_starts_that_do_not_ascend_stay_within_the_workspace(ctx, starts):
    """Rows that overlap make more segments than the workspace holds: nothing behind it is written, and the first
    sequence whose starts descend is reported."""
    k = kvx()
    t, heads, p, n = 3000, 2, 128, 128
    s = len(starts) - 1
    wide, x, b, c, dt, A, D, dt_bias = scan_inputs(t, heads, p, n, 1, BF16)
    st = Slots(s, heads, p, n)
    batch = k.StateBatch(ints(list(range(s))), starts=ints(starts), tokens=t)
    need = k.kv_state_scan_workspace(ctx, batch, heads, p, n).numel()
    room = torch.full((need + s * 24 * heads * p * n * 4,), 0xA5, dtype=torch.uint8, device="cuda")  # as many as overlapping rows make
    out = torch.empty((t, heads, p), dtype=BF16, device="cuda")
    k.kv_state_scan(ctx, st.slots, batch, x.cuda(), dt.cuda(), A.cuda(), b.cuda(), c.cuda(), out, workspace=room[:need])
    torch.cuda.synchronize()
    assert bool((room[need:] == 0xA5).all())
    assert k.kv_get_device_error(ctx) == next(i for i in range(s) if starts[i + 1] < starts[i])
    k.kv_state_conv(ctx, st.slots, batch, normal((t, 8), BF16, 8).cuda(), normal((8, 4), BF16, 9).cuda(),
                    torch.empty((t, 8), dtype=BF16, device="cuda"))
    torch.cuda.synchronize()
    assert k.kv_get_device_error(ctx) == next(i for i in range(s) if starts[i + 1] < starts[i])


@pytest.mark.parametrize("t", [10, 300, 3000])
def test_starts_past_the_rows_are_cut_and_reported(ctx, t):
    k = kvx()
    heads, p, n = 2, 64, 64
    wide, x, b, c, dt, A, D, dt_bias = scan_inputs(t, heads, p, n, 1, BF16)
    dev = [v.cuda() for v in (x, dt, A, b, c)]
    xc, w = normal((t, 8), BF16, 8).cuda(), normal((8, 4), BF16, 9).cuda()
    got = []
    for starts, bad in (([0, 7, t], -1), ([0, 7, t + 500], 1), ([-3, 7, 2 ** 31 - 1], 0)):
        st = Slots(2, heads, p, n)
        batch = k.StateBatch(ints([0, 1]), starts=ints(starts), tokens=t)
        out, cv = torch.zeros((t, heads, p), dtype=BF16, device="cuda"), torch.zeros((t, 8), dtype=BF16, device="cuda")
        k.kv_state_scan(ctx, st.slots, batch, dev[0], dev[1], dev[2], dev[3], dev[4], out,
                        workspace=k.kv_state_scan_workspace(ctx, batch, heads, p, n))
        torch.cuda.synchronize()
        assert k.kv_get_device_error(ctx) == bad
        k.kv_state_conv(ctx, st.slots, batch, xc, w, cv)
        torch.cuda.synchronize()
        assert k.kv_get_device_error(ctx) == bad
        got.append((out, cv, st.dev))
    for g in got[1:]:
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(g, got[0]))


@pytest.mark.parametrize("t,heads", [(100, 2), (3000, 2)])
def test_wait_for_the_tensor_cores_runs_out_then_recovery(t, heads):
    """Fault point "scan_wait": the end of the first chunk's products is not announced, so the wait for it (2e6 cycles
    here) runs out.  The call returns, kv_get_device_error tells, and the next call on the context is right."""
    k = kvx()
    p, n = 128, 64
    wide, x, b, c, dt, A, D, dt_bias = scan_inputs(t, heads, p, n, 1, BF16)
    batch, _ = batch_of([t], [0])
    c2 = k.kv_ctx_create(0, wait_cycles=2_000_000)
    try:
        dev = [v.cuda() for v in (x, dt, A, b, c)]
        outs = []
        for fault in (True, False):
            st = Slots(1, heads, p, n)
            out = torch.zeros((t, heads, p), dtype=BF16, device="cuda")
            ws = k.kv_state_scan_workspace(c2, batch, heads, p, n)
            torch.cuda.synchronize()
            if fault:
                k.kv_fault_inject("scan_wait")
            k.kv_state_scan(c2, st.slots, batch, dev[0], dev[1], dev[2], dev[3], dev[4], out, workspace=ws)
            torch.cuda.synchronize()
            if fault:
                with pytest.raises(k.KvxError) as e:
                    k.kv_get_device_error(c2)
                assert e.value.status == k.KVX_ETIMEOUT
            assert k.kv_get_device_error(c2) == -1
            outs.append(out)
        y, _, size, _ = refs.scan(x.double(), dt.double(), A.double(), b.double(), c.double(), None, None, True, st.state[0].double())
        assert bool(((outs[1].cpu().double() - y).abs() <= refs.UNIT[BF16] * y.abs() + (3 * refs.UNIT[BF16] + 2.0 ** -13) * size + 1e-7).all())
    finally:
        k.kv_fault_inject(None)
        k.kv_ctx_destroy(c2)


def test_without_the_matrix_form_everything_still_works():
    """Fault point "scan_setup": a context whose matrix form cannot be used, as with kernels compiled for fewer
    registers, is made all the same, moves slots and scans prompts token by token."""
    k = kvx()
    k.kv_fault_inject("scan_setup")
    c = k.kv_ctx_create(0)
    try:
        check_scan(c, [300, 0, 17, 40], 2, 128, 128, 1, BF16)
        check_scan(c, [1, 1], 2, 128, 128, 1, FP16, single=True)
        batch, _ = batch_of([3000], [0])
        assert k.kv_state_scan_workspace(c, batch, 2, 128, 128).numel() == 16  # the least there is
        before = k.kv_ctx_stats(c)["kernel_launches"]
        st = Slots(1, 2, 64, 64)
        batch, _ = batch_of([500], [0])
        wide, x, b, cc, dt, A, D, dt_bias = scan_inputs(500, 2, 64, 64, 1, BF16)
        out = torch.empty((500, 2, 64), dtype=BF16, device="cuda")
        k.kv_state_scan(c, st.slots, batch, x.cuda(), dt.cuda(), A.cuda(), b.cuda(), cc.cuda(), out)
        assert k.kv_ctx_stats(c)["kernel_launches"] == before + 1
        host = k.HostBuffer(st.bytes)
        k.kv_state_store(c, [st.dev.view(-1)], 1, st.bytes, 0, host.tensor)
        torch.cuda.synchronize()
        assert torch.equal(host.tensor[:st.bytes], st.dev.cpu()[0])
        host.close()
    finally:
        k.kv_fault_inject(None)
        k.kv_ctx_destroy(c)
    c = k.kv_ctx_create(0)  # and the next context has it
    try:
        batch, _ = batch_of([3000], [0])
        assert k.kv_state_scan_workspace(c, batch, 2, 128, 128).numel() > 16
    finally:
        k.kv_ctx_destroy(c)


def test_captured_step(ctx):
    """A captured convolution and scan of single tokens, replayed: the state moves on in its slot."""
    k = kvx()
    heads, p, n = 2, 64, 64
    st = Slots(2, heads, p, n, channels=64)
    batch = k.StateBatch(ints([1]))
    wide, x, b, c, dt, A, D, dt_bias = scan_inputs(3, heads, p, n, 1, BF16)
    bufs = [v[:1].cuda() for v in (x, dt, b, c)]
    cx, w = normal((3, 64), BF16, 8), normal((64, 4), BF16, 9)
    cbuf, wd, Ad, out, cout = cx[:1].cuda(), w.cuda(), A.cuda(), torch.empty((1, heads, p), dtype=BF16, device="cuda"), torch.empty((1, 64), dtype=BF16, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        k.kv_state_conv(ctx, st.slots, batch, cbuf, wd, cout)
        k.kv_state_scan(ctx, st.slots, batch, bufs[0], bufs[1], Ad, bufs[2], bufs[3], out)
    y, state, size, big = refs.scan(x.double(), dt.double(), A.double(), b.double(), c.double(), None, None, True, st.state[1].double())
    cy, window = refs.conv(cx.double(), w.double(), None, st.window[1].double(), True)
    for i in range(3):
        for buf, v in zip(bufs + [cbuf], (x, dt, b, c, cx)):
            buf.copy_(v[i:i + 1])
        graph.replay()
        torch.cuda.synchronize()
        assert bool(((out[0].cpu().double() - y[i]).abs() <= refs.UNIT[BF16] * y[i].abs() + 2.0 ** -13 * size[i] + 1e-7).all())
        assert bool(((cout[0].cpu().double() - cy[i]).abs() <= refs.UNIT[BF16] * cy[i].abs() + 1e-5).all())
    assert bool(((st.dev.cpu()[1, :st.rec].view(torch.float32).view(heads, p, n).double() - state).abs() <= 2.0 ** -14 * big).all())
    assert torch.equal(st.dev.cpu()[1, st.rec:st.rec + st.win].view(BF16).view(3, 64).double(), window)
    assert torch.equal(st.dev.cpu()[0], st.cpu[0])


def test_slots_past_four_gib(ctx):
    k = kvx()
    slot = 64 << 10
    n = (5 << 30) // slot
    buf = torch.zeros(n * slot, dtype=torch.uint8, device="cuda")
    slots = k.StateSlots(buf, n, slot, 0, 32 << 10)
    batch = k.StateBatch(ints([n - 1]))
    wide, x, b, c, dt, A, D, dt_bias = scan_inputs(1, 2, 64, 64, 1, BF16)
    out = torch.empty((1, 2, 64), dtype=BF16, device="cuda")
    k.kv_state_scan(ctx, slots, batch, x.cuda(), dt.cuda(), A.cuda(), b.cuda(), c.cuda(), out)
    torch.cuda.synchronize()
    _, state, _, big = refs.scan(x.double(), dt.double(), A.double(), b.double(), c.double(), None, None, True,
                                 torch.zeros((2, 64, 64), dtype=torch.float64))
    got = buf.view(n, slot)[n - 1, :32 << 10].view(torch.float32).view(2, 64, 64).cpu().double()
    assert bool(((got - state).abs() <= 2.0 ** -14 * big + 1e-9).all())
    assert int(buf.view(n, slot)[:n - 1].max()) == 0


def test_refusals(ctx):
    k = kvx()
    st = Slots(2, 2, 64, 64, channels=64)
    batch = k.StateBatch(ints([0, 1]))
    wide, x, b, c, dt, A, D, dt_bias = scan_inputs(2, 2, 64, 64, 1, BF16)
    x, b, c, dt, A = (v.cuda() for v in (x, b, c, dt, A))
    out = torch.full((2, 2, 64), 7.0, dtype=BF16, device="cuda")

    def scan(status, slots=st.slots, batch=batch, x=x, dt=dt, b=b, c=c, out=out, A=A, **kw):
        with pytest.raises(k.KvxError) as e:
            k.kv_state_scan(ctx, slots, batch, x, dt, A, b, c, out, **kw)
        assert e.value.status == status, e.value

    scan(k.KVX_EINVAL, b=b[..., :48], c=c[..., :48])
    scan(k.KVX_EALIGN, x=x[..., :60], out=out[..., :60])
    scan(k.KVX_ERANGE, slots=k.StateSlots(st.dev, 2, st.bytes, st.bytes - 16, 0))
    scan(k.KVX_EALIGN, slots=k.StateSlots(st.dev, 2, st.bytes, 8, 0))
    scan(k.KVX_EINVAL, slots=k.StateSlots(st.dev, 0, st.bytes, 0, 0))
    scan(k.KVX_EDEVICE, x=x.cpu())
    scan(k.KVX_EDEVICE, A=A.cpu())
    scan(k.KVX_EINVAL, out=out[:1].expand(2, 2, 64))
    w, xc = normal((64, 4), BF16, 9).cuda(), normal((2, 64), BF16, 8).cuda()
    co = torch.full((2, 64), 7.0, dtype=BF16, device="cuda")

    def conv(status, slots=st.slots, x=xc, w=w, out=co, **kw):
        with pytest.raises(k.KvxError) as e:
            k.kv_state_conv(ctx, slots, batch, x, w, out, **kw)
        assert e.value.status == status, e.value

    conv(k.KVX_EINVAL, w=torch.zeros((64, 5), dtype=BF16, device="cuda"))
    conv(k.KVX_EALIGN, w=w[:60], x=xc[:, :60], out=co[:, :60])
    conv(k.KVX_ERANGE, slots=k.StateSlots(st.dev, 2, st.bytes, 0, st.bytes - 16))
    conv(k.KVX_EDEVICE, out=co.cpu())
    assert bool((out == 7.0).all()) and bool((co == 7.0).all())
    assert torch.equal(st.dev.cpu(), st.cpu)
    with pytest.raises(ValueError):
        k.StateBatch(ints([0]), starts=ints([0, 4]))
    with pytest.raises(TypeError):
        k.StateBatch(ints([0]).long())
    with pytest.raises(ValueError):
        k.kv_state_scan(ctx, st.slots, batch, x[:1], dt, A, b, c, out)
