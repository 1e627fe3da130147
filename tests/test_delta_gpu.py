"""kv_state_delta against a token-by-token 64-bit recurrence, and the mixers of a hybrid model's step together."""
import math

import pytest
import torch

import mixer_refs as mixers
import operator_refs as refs
from gpu_util import kvx
from test_state_ops_gpu import Slots, batch_of, ints, normal

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    k = kvx()
    c = k.kv_ctx_create(0)
    yield c
    k.kv_ctx_destroy(c)


class Inputs:
    """What a recurrent layer's projections and its convolution (past a SiLU) put out, within one tensor."""

    def __init__(self, t, heads, p, n, groups, dtype, seed=3, decay=1.0):
        wide = torch.nn.functional.silu(normal((t, 2 * groups * n + heads * p + 8), torch.float32, seed, 1.5)).to(dtype)
        self.wide, self.gates = wide, normal((t, 2 * heads + 3), dtype, seed + 1)
        self.heads, self.p, self.n, self.groups = heads, p, n, groups
        g = torch.Generator().manual_seed(seed + 2)
        self.A = -(1.0 + 15.0 * torch.rand(heads, generator=g)) * decay
        step = torch.exp(torch.rand(heads, generator=g) * math.log(100.0) + math.log(1e-3))
        self.bias = torch.log(torch.expm1(step))

    def of(self, wide, gates):
        t, a = wide.shape[0], self.groups * self.n
        return {"query": wide[:, :a].view(t, self.groups, self.n), "key": wide[:, a:2 * a].view(t, self.groups, self.n),
                "value": wide[:, 2 * a:2 * a + self.heads * self.p].view(t, self.heads, self.p),
                "dt": gates[:, :self.heads], "beta": gates[:, self.heads:2 * self.heads]}

    def cpu(self):
        return self.of(self.wide, self.gates)

    def cuda(self):
        return self.of(self.wide.cuda(), self.gates.cuda())


def close(got, want, got_state, state, slack, terms, q, dtype, products):
    """Whether outputs and state are as near as roundings in 32 bits, and of the product form's factors, let them be.

    A step's numbers are rounded a few times in 32 bits, sums of up to 256 terms by trees of four to 32 partial sums, factors
    of matrices split to 22 bits or more: less than 2^-18 of what is added up.  The product form of the outputs
    rounds both factors of a term (and in fp16 a scaled one, of 2^-14 at least) to the inputs' type."""
    unit, rows = refs.UNIT[dtype], want.shape[0]
    per_row = 2.0 ** -18 * slack
    size = torch.linalg.vector_norm(q, dim=-1)[:rows, :, None]
    bound = unit * want.abs() + per_row[1:] * size + (2.5 * unit * terms if products else 0) + 2.0 ** -25
    off = (got - want).abs()
    assert bool((off <= bound).all()), float((off / bound).max())
    off = torch.linalg.vector_norm(got_state - state, dim=-1)
    assert bool((off <= per_row[-1] + 1e-9).all()), float((off / (per_row[-1] + 1e-9)).max())


def check(ctx, lens, heads, p, n, groups, dtype, single=False, in_place=False, fresh=None, decayed=True, bias=True, softplus=True,
          sigmoid=True, normalize=True, scale=None, decay=1.0, stream=None, change=None):
    k = kvx()
    s = len(lens)
    st = Slots(2 * s + 1, heads, p, n, dtype=dtype)
    ins = list(range(s)) if in_place else list(range(s, 0, -1))
    outs = ins if in_place else [s + 1 + i for i in range(s)]
    batch, starts = batch_of(lens, ins, None if in_place else outs, fresh, single)
    t = starts[-1]
    data = Inputs(t, heads, p, n, groups, dtype, decay=decay)
    if not softplus:
        data.gates[:, :heads] = data.gates[:, :heads].abs() * 0.02
    if not sigmoid:
        data.gates[:, heads:] = torch.rand((t, heads + 3), generator=torch.Generator().manual_seed(9)).to(dtype)
    if not normalize:
        data.wide *= 1 / math.sqrt(n)
    if change:
        change(data)
    x, cpu = data.cuda(), data.cpu()
    out = torch.full((t, heads * p + 8), 7.0, dtype=dtype, device="cuda")
    ws = k.kv_state_delta_workspace(ctx, batch, heads, p, n)
    ws.fill_(0xFF)
    options = dict(softplus=softplus, sigmoid=sigmoid, normalize=normalize, scale=scale)
    given = dict(A=data.A.cuda(), dt_bias=data.bias.cuda() if bias else None)
    if not decayed:
        x.pop("dt"), given.clear()
    torch.cuda.synchronize()
    k.kv_state_delta(ctx, st.slots, batch, out=out[:, :heads * p].view(t, heads, p), workspace=ws, stream=stream, **x, **given, **options)
    torch.cuda.synchronize()
    got_state = st.dev.cpu()[:, :st.rec].view(torch.float32).view(st.state.shape)
    untouched = st.cpu.clone()
    for i in range(s):
        rows = slice(starts[i], starts[i + 1])
        first = torch.zeros_like(st.state[0]) if fresh and fresh[i] else st.state[ins[i]]
        y, state, slack, terms, q = mixers.delta(cpu["query"][rows], cpu["key"][rows], cpu["value"][rows], cpu["beta"][rows], first,
                                                 cpu["dt"][rows] if decayed else None, data.A, data.bias if bias else None, **options)
        got = out[rows, :heads * p].view(-1, heads, p).cpu().double()
        close(got, y, got_state[outs[i]].double(), state, slack, terms, q, dtype, lens[i] > 1)
        untouched[outs[i], :st.rec] = st.dev.cpu()[outs[i], :st.rec]
    assert bool((out[:, heads * p:] == 7.0).all())
    assert torch.equal(st.dev.cpu(), untouched)
    assert k.kv_get_device_error(ctx) == -1


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("p", [8, 64, 120, 128, 256])
@pytest.mark.parametrize("n", [16, 32, 64, 128, 256])
def test_single_tokens(ctx, dtype, p, n):
    check(ctx, [1, 1, 1], 4, p, n, 2, dtype, single=True, in_place=n == 64)


def test_single_tokens_of_many_sequences(ctx):
    check(ctx, [1] * 70, 8, 128, 128, 4, BF16, single=True)


# lengths around the 64 tokens of a chunk, of one token and of none
LENS = [0, 1, 2, 63, 64, 65, 127, 128, 129, 300]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("p,n,heads,groups", [(64, 64, 2, 1), (64, 128, 4, 2), (128, 64, 3, 3), (128, 128, 2, 1)])
def test_prompts(ctx, dtype, p, n, heads, groups):
    check(ctx, LENS, heads, p, n, groups, dtype)
    check(ctx, [200, 5], heads, p, n, groups, dtype, in_place=True, fresh=[1, 0])


@pytest.mark.parametrize("p,n", [(8, 16), (40, 32), (256, 64), (64, 256), (72, 128), (16, 16), (24, 64), (8, 128)])
def test_prompts_of_other_sizes(ctx, p, n):
    check(ctx, [0, 1, 40, 150], 2, p, n, 1, BF16)


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_short_and_long_sequences_together(ctx, dtype):
    check(ctx, [17, 16, 15, 0, 400, 1], 2, 128, 128, 1, dtype, fresh=[0, 1, 0, 0, 1, 0])
    check(ctx, [17, 0, 1, 16, 3, 1, 2, 2], 2, 128, 128, 1, dtype, fresh=[0, 1, 0, 0, 1, 0, 0, 0])
    check(ctx, [3, 16, 17, 0, 2] * 7 + [200, 1, 90], 2, 64, 64, 2, dtype, in_place=True)
    check(ctx, [1] * 20, 2, 64, 64, 2, dtype)


@pytest.mark.parametrize("t", [1, 2, 15, 16, 17, 33, 48, 64, 384, 520])
def test_one_sequence(ctx, t):
    check(ctx, [t], 3, 128, 128, 1, BF16)


def test_long_prompts(ctx):
    check(ctx, [1500, 700], 2, 128, 128, 1, BF16)
    check(ctx, [2100], 1, 64, 128, 1, FP16)


def test_a_prompt_in_fp16_is_off_by_its_rounding(ctx):
    """Factors in two parts are off by 2^-22, sums by some 2^-20: beside the rounding of an output, 2^-11 at most and
    2^-11 / sqrt(3) in the mean square, they are nothing.  (A factor rounded to fp16 once would add half of that to the square.)"""
    k = kvx()
    t, heads, n = 700, 2, 128
    st = Slots(2, heads, n, n, dtype=FP16)
    batch, _ = batch_of([t], [0], [1], [1], False)
    data = Inputs(t, heads, n, n, 1, FP16, seed=31)
    out = torch.empty((t, heads, n), dtype=FP16, device="cuda")
    k.kv_state_delta(ctx, st.slots, batch, out=out, A=data.A.cuda(), dt_bias=data.bias.cuda(),
                     workspace=k.kv_state_delta_workspace(ctx, batch, heads, n, n), **data.cuda())
    torch.cuda.synchronize()
    x = data.cpu()
    y = mixers.delta(x["query"], x["key"], x["value"], x["beta"], torch.zeros_like(st.state[0]), x["dt"], data.A, data.bias)[0]
    rounding, off = y.half().double() - y, out.cpu().double() - y
    assert float(off.square().mean()) <= 1.1 * float(rounding.square().mean())


@pytest.mark.parametrize("t,n", [(700, 128), (60, 64)])
def test_a_prompt_in_bf16_is_off_by_its_rounding(ctx, t, n):
    """As in fp16: what the factors' 2^-22 and the sums' 2^-20 or so of an output's terms add to the square of its rounding, 2^-9 to 2^-8
    of it, is below 2^-20 of that even where the terms are 2^3 times the output.  (Factors rounded to fp16 once, 2^-11 at most
    and half of that in the root mean square for either, would add some 2 % to the square.)"""
    k = kvx()
    heads = 2
    st = Slots(2, heads, n, n, dtype=BF16)
    batch, _ = batch_of([t], [0], [1], [1], False)
    data = Inputs(t, heads, n, n, 1, BF16, seed=32)
    out = torch.empty((t, heads, n), dtype=BF16, device="cuda")
    k.kv_state_delta(ctx, st.slots, batch, out=out, A=data.A.cuda(), dt_bias=data.bias.cuda(),
                     workspace=k.kv_state_delta_workspace(ctx, batch, heads, n, n), **data.cuda())
    torch.cuda.synchronize()
    x = data.cpu()
    y = mixers.delta(x["query"], x["key"], x["value"], x["beta"], torch.zeros_like(st.state[0]), x["dt"], data.A, data.bias)[0]
    rounding, off = y.bfloat16().double() - y, out.cpu().double() - y
    assert float(off.square().mean()) <= 1.002 * float(rounding.square().mean())


@pytest.mark.parametrize("softplus,sigmoid,normalize,bias", [(False, True, True, False), (True, False, True, True), (True, True, False, False),
                                                             (False, False, False, False)])
def test_options(ctx, softplus, sigmoid, normalize, bias):
    for dtype in (BF16, FP16):
        check(ctx, [150, 1, 30], 2, 64, 128, 1, dtype, softplus=softplus, sigmoid=sigmoid, normalize=normalize, bias=bias, scale=0.3,
              stream=torch.cuda.Stream())


def test_without_decay(ctx):
    check(ctx, [200, 1, 20], 2, 64, 64, 1, BF16, decayed=False)
    check(ctx, [1, 1], 2, 64, 64, 1, FP16, decayed=False, single=True)


@pytest.mark.parametrize("decay", [1e-4, 30.0, 1000.0])
def test_slow_and_fast_decays(ctx, decay):
    """From states that forget nothing to ones that forget within a token."""
    check(ctx, [260, 70], 4, 64, 64, 1, BF16, decay=decay, bias=decay < 1)


def test_slow_decays_behind_fast_ones(ctx):
    """A decay is taken of the tokens between two, however large the exponents before them are."""
    def change(data):
        data.A[:] = -torch.tensor([8.0, 80.0, 800.0, 8e6])
        slow = torch.tensor([1e-5, 5e-6, 5e-6, 1e-7])
        data.gates[:, :4] = torch.where(torch.arange(128)[:, None] % 64 < 32, torch.tensor(3.0), slow).to(data.gates.dtype)
    check(ctx, [128], 4, 64, 64, 1, BF16, change=change, softplus=True, bias=False)


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_equal_keys_and_full_steps(ctx, dtype):
    """Keys that are all the same, written with full steps: a token's value takes the place of the one before."""
    def change(data):
        t = data.wide.shape[0]
        data.wide[:, :2 * data.groups * data.n] = data.wide[:1, :2 * data.groups * data.n].expand(t, -1)
        data.gates[:, data.heads:] = 30.0
    check(ctx, [300, 64], 2, 64, 128, 1, dtype, change=change, decayed=False)


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_rows_of_small_and_large_numbers(ctx, dtype):
    """Keys and queries are taken to unit length whatever they are, and rows of zeros stay zeros; values from small to large, a row
    of the state each."""
    def change(data):
        a = data.groups * data.n
        sizes = torch.exp2(torch.arange(data.wide.shape[0]).float() % 14 - 7)[:, None]
        data.wide[:, :2 * a] = (data.wide[:, :2 * a] * sizes).to(dtype)
        data.wide[3::10, :2 * a] = 0
        data.wide[:, 2 * a:2 * a + data.heads * data.p] *= torch.exp2(torch.arange(data.p).float() % 18 - 9).repeat(data.heads).to(dtype)
    check(ctx, [200, 65], 2, 64, 128, 1, dtype, change=change)


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_steps_that_make_the_state_grow(ctx, dtype):
    """Keys that are not of unit length with b |k|^2 above 2: the recurrence itself grows, and is followed."""
    k = kvx()
    t, heads, p, n = 96, 2, 64, 64
    data = Inputs(t, heads, p, n, 1, dtype, seed=11)
    data.wide[:, n:2 * n] = (data.wide[:, n:2 * n] * 0.21).to(dtype)  # |k|^2 about 5
    st = Slots(1, heads, p, n, dtype=dtype)
    batch, _ = batch_of([t], [0])
    out = torch.empty((t, heads, p), dtype=dtype, device="cuda")
    k.kv_state_delta(ctx, st.slots, batch, out=out, A=data.A.cuda() * 0.01, normalize=False,
                     workspace=k.kv_state_delta_workspace(ctx, batch, heads, p, n), **data.cuda())
    x = data.cpu()
    y, state, _, _, _ = mixers.delta(x["query"], x["key"], x["value"], x["beta"], st.state[0], x["dt"], data.A * 0.01, normalize=False)
    after = st.dev.cpu()[0, :st.rec].view(torch.float32).view(state.shape).double()
    # a rounding of 2^-18 a step grows as the state does
    assert float((after - state).norm()) <= t * 2.0 ** -18 * float(state.norm())
    fine = y.abs() < 60000
    assert bool(fine.any())
    size = y.abs().cummax(0)[0].amax(-1, keepdim=True)
    assert bool(((out.cpu().double() - y).abs()[fine] <= ((6 * refs.UNIT[dtype] + t * 2.0 ** -16) * size + 1e-3).expand_as(y)[fine]).all())


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("p,n", [(64, 64), (128, 128), (8, 32)])
def test_infinities_and_nan_reach_nothing_before_them(ctx, dtype, p, n):
    """A value's reach its own row of the state from its token on, a key's the whole head's; nothing before changes."""
    k = kvx()
    t, heads = 300, 3
    data = Inputs(t, heads, p, n, 3, dtype)
    clean, x = data.cpu(), Inputs(t, heads, p, n, 3, dtype)
    y = x.cpu()
    y["value"][70, 0, 3], y["value"][150, 0, 5], y["key"][200, 1, 2], y["query"][250, 2, 1] = math.inf, math.nan, math.inf, math.nan
    outs, states = [], []
    for d in (data, x):
        st = Slots(1, heads, p, n, dtype=dtype)
        batch, _ = batch_of([t], [0])
        out = torch.empty((t, heads, p), dtype=dtype, device="cuda")
        k.kv_state_delta(ctx, st.slots, batch, out=out, A=d.A.cuda(), workspace=k.kv_state_delta_workspace(ctx, batch, heads, p, n), **d.cuda())
        outs.append(out.cpu().double()), states.append(st.dev.cpu()[0, :st.rec].view(torch.float32).view(heads, p, n))
    fine = torch.ones((t, heads, p), dtype=torch.bool)
    fine[70:, 0, 3] = fine[150:, 0, 5] = fine[200:, 1] = fine[250, 2] = False
    assert torch.equal(torch.isfinite(outs[1]), fine)
    want, _, slack, terms, q = mixers.delta(clean["query"], clean["key"], clean["value"], clean["beta"], st.state[0], clean["dt"], data.A)
    size = torch.linalg.vector_norm(q, dim=-1)[:, :, None]
    bound = refs.UNIT[dtype] * (want.abs() + 2.5 * terms) + 2.0 ** -18 * slack[1:] * size + 2.0 ** -25
    assert bool(((outs[1] - want).abs()[fine] <= bound[fine]).all())
    rows = torch.isfinite(states[1]).all(-1)
    assert rows[2].all() and not rows[1].any() and (~rows[0]).nonzero().flatten().tolist() == [3, 5]


def test_fresh_sequences_do_not_read_their_slots(ctx):
    k = kvx()
    for lens, single in (([1, 1], True), ([130, 3], False)):
        st = Slots(2, 2, 64, 64)
        st.dev.fill_(0xFF)
        batch, starts = batch_of(lens, [1, 0], fresh=[1, 1], single=single)
        data = Inputs(starts[-1], 2, 64, 64, 1, BF16)
        out = torch.empty((starts[-1], 2, 64), dtype=BF16, device="cuda")
        k.kv_state_delta(ctx, st.slots, batch, out=out, A=data.A.cuda(), workspace=k.kv_state_delta_workspace(ctx, batch, 2, 64, 64), **data.cuda())
        assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(st.dev[:, :st.rec].view(torch.float32)).all())


def test_token_by_token_is_the_prompt(ctx):
    """A prompt's state and last output are those of its tokens one by one, within the roundings of both."""
    k = kvx()
    t, heads, p, n = 200, 2, 64, 128
    data = Inputs(t, heads, p, n, 1, BF16)
    x, A = data.cuda(), data.A.cuda()
    one, all_ = Slots(1, heads, p, n), Slots(1, heads, p, n)
    batch, _ = batch_of([t], [0])
    out = torch.empty((t, heads, p), dtype=BF16, device="cuda")
    k.kv_state_delta(ctx, all_.slots, batch, out=out, A=A, workspace=k.kv_state_delta_workspace(ctx, batch, heads, p, n), **x)
    single, _ = batch_of([1], [0], single=True)
    last = torch.empty((1, heads, p), dtype=BF16, device="cuda")
    for i in range(t):
        k.kv_state_delta(ctx, one.slots, single, out=last, A=A, **{name: v[i:i + 1] for name, v in x.items()})
    torch.cuda.synchronize()
    c = data.cpu()
    y, state, slack, terms, q = mixers.delta(c["query"], c["key"], c["value"], c["beta"], one.state[0], c["dt"], data.A)
    for got, st, products in ((last, one, False), (out[-1:], all_, True)):
        after = st.dev.cpu()[0, :st.rec].view(torch.float32).view(state.shape).double()
        close(got.cpu().double(), y[-1:], after, state, slack[-2:], terms[-1:], q[-1:], BF16, products)


def test_bad_slots_give_zeros_and_are_reported(ctx):
    k = kvx()
    for lens, single in (([1, 1, 1], True), ([3, 100, 70], False), ([3, 2, 1], False)):
        st = Slots(3, 2, 64, 64)
        batch, starts = batch_of(lens, [0, 3, 2], [0, 1, -1], single=single)
        data = Inputs(starts[-1], 2, 64, 64, 1, BF16)
        out = torch.full((starts[-1], 2, 64), 7.0, dtype=BF16, device="cuda")
        k.kv_state_delta(ctx, st.slots, batch, out=out, A=data.A.cuda(), workspace=k.kv_state_delta_workspace(ctx, batch, 2, 64, 64), **data.cuda())
        torch.cuda.synchronize()
        assert bool((out[starts[1]:] == 0).all()) and not bool((out[:starts[1]] == 0).all())
        assert torch.equal(st.dev.cpu()[1:], st.cpu[1:])
        assert k.kv_get_device_error(ctx) == 1


@pytest.mark.parametrize("starts", [[0, 100, 50, 200], [0, 200, 0, 200], [150, 200, 0, 90], [0, 90, 500, 200], [-5, 30, 60, 90], [40, 60, 100, 190]])
def test_starts_that_do_not_ascend_stay_within_the_rows(ctx, starts):
    """Cut to the rows there are and reported; rows in no sequence are left as they were."""
    k = kvx()
    t, s = 200, 3
    st = Slots(2 * s, 2, 64, 64)
    data = Inputs(t, 2, 64, 64, 1, BF16)
    batch = k.StateBatch(ints([0, 1, 2]), ints([3, 4, 5]), starts=ints(starts), tokens=t)
    wide = torch.full((t + 40, 2, 64), 7.0, dtype=BF16, device="cuda")
    ws = k.kv_state_delta_workspace(ctx, batch, 2, 64, 64)
    guarded = torch.full((ws.numel() + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    k.kv_state_delta(ctx, st.slots, batch, out=wide[20:20 + t], A=data.A.cuda(), workspace=guarded[:ws.numel()], **data.cuda())
    torch.cuda.synchronize()
    assert bool((wide[:20] == 7.0).all()) and bool((wide[20 + t:] == 7.0).all()) and bool((guarded[ws.numel():] == 0x5A).all())
    covered = torch.zeros(t, dtype=torch.bool)
    for a, b in zip(starts, starts[1:]):
        covered[max(a, 0):max(min(b, t), max(a, 0))] = True
    assert bool((wide[20:20 + t].cpu()[~covered] == 7.0).all())
    bad = any(a < 0 or b < a or b > t for a, b in zip(starts, starts[1:]))
    assert (k.kv_get_device_error(ctx) != -1) == bad


def test_wait_for_a_copy_runs_out_then_recovery():
    """The second chunk's copies are left out: the walk gives up after its limit, reports it and writes no state."""
    k = kvx()
    c = k.kv_ctx_create(0, wait_cycles=2_000_000)
    try:
        t, heads, p, n = 200, 2, 64, 64
        data = Inputs(t, heads, p, n, 1, BF16)
        x, A = data.cuda(), data.A.cuda()
        batch, _ = batch_of([t], [0], [1])
        outs = []
        for point in (None, "delta_wait", None):
            st = Slots(2, heads, p, n)
            out = torch.zeros((t, heads, p), dtype=BF16, device="cuda")
            if point:
                k.kv_fault_inject(point)
            k.kv_state_delta(c, st.slots, batch, out=out, A=A, workspace=k.kv_state_delta_workspace(c, batch, heads, p, n), **x)
            torch.cuda.synchronize()
            if point:
                assert torch.equal(st.dev.cpu(), st.cpu)
                with pytest.raises(k.KvxError) as e:
                    k.kv_get_device_error(c)
                assert e.value.status == k.KVX_ETIMEOUT
            else:
                outs.append((out, st.dev))
                assert k.kv_get_device_error(c) == -1
        assert all(torch.equal(a, b) for a, b in zip(*outs))
    finally:
        k.kv_ctx_destroy(c)


@pytest.mark.parametrize("t, odd", [(200, False), (50, False), (200, True)])
def test_wait_for_what_the_outputs_take_runs_out_then_recovery(t, odd):
    """The first chunk's factors of the outputs are left out, by chunks and token by token, of several chunks and of one: every
    warp ends before the next chunk's are asked for, no state is written, and the next call gives what the first gave."""
    k = kvx()
    c = k.kv_ctx_create(0, wait_cycles=2_000_000)
    try:
        heads, p, n = 2, 64, 64
        data = Inputs(t, heads, p, n, 1, BF16)
        x, A = data.cuda(), data.A.cuda()
        if odd:
            x["value"][5, 0, 3] = math.inf
        batch, _ = batch_of([t], [0], [1])
        outs = []
        for point in (None, "delta_wait_m", None):
            st = Slots(2, heads, p, n)
            out = torch.zeros((t, heads, p), dtype=BF16, device="cuda")
            if point:
                k.kv_fault_inject(point)
            k.kv_state_delta(c, st.slots, batch, out=out, A=A, workspace=k.kv_state_delta_workspace(c, batch, heads, p, n), **x)
            torch.cuda.synchronize()
            if point:
                assert torch.equal(st.dev.cpu(), st.cpu)
                assert not bool(out[64:].any())  # chunks that were not begun
                with pytest.raises(k.KvxError) as e:
                    k.kv_get_device_error(c)
                assert e.value.status == k.KVX_ETIMEOUT
            else:
                outs.append((out.view(torch.int16), st.dev))
                assert k.kv_get_device_error(c) == -1
        assert all(torch.equal(a, b) for a, b in zip(*outs))
    finally:
        k.kv_ctx_destroy(c)


def test_captured_step(ctx):
    """Replayed with other slots, starts and freshness, on a workspace that calls in between have used."""
    k = kvx()
    heads, p, n, t = 2, 64, 64, 150
    st = Slots(4, heads, p, n)
    data = Inputs(t, heads, p, n, 1, BF16)
    x, A = data.cuda(), data.A.cuda()
    slots, starts, fresh = ints([0, 1]), ints([0, 100, t]), ints([0, 0])
    batch = k.StateBatch(slots, ints([2, 3]), starts=starts, tokens=t, fresh=fresh)
    out = torch.zeros((t, heads, p), dtype=BF16, device="cuda")
    ws = k.kv_state_delta_workspace(ctx, batch, heads, p, n)
    run = lambda: k.kv_state_delta(ctx, st.slots, batch, out=out, A=A, workspace=ws, **x)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for a, b, c in (([1, 0], [0, 3, t], [0, 1]), ([0, 1], [0, 0, t], [1, 0]), ([1, 0], [0, 64, 128], [0, 0])):
        slots.copy_(ints(a)), starts.copy_(ints(b)), fresh.copy_(ints(c))
        ws.fill_(0xFF)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), st.dev.clone()
        out.zero_()
        run()
        torch.cuda.synchronize()
        assert torch.equal(out, got[0]) and torch.equal(st.dev, got[1])


def test_same_bits_every_time(ctx):
    k = kvx()
    lens, heads = [500, 3, 77], 2
    data = Inputs(580, heads, 128, 128, 1, FP16)
    x, A = data.cuda(), data.A.cuda()
    runs = []
    for _ in range(3):
        st = Slots(6, heads, 128, 128, dtype=FP16)
        batch, _ = batch_of(lens, [0, 1, 2], [3, 4, 5])
        out = torch.empty((580, heads, 128), dtype=FP16, device="cuda")
        k.kv_state_delta(ctx, st.slots, batch, out=out, A=A, workspace=k.kv_state_delta_workspace(ctx, batch, heads, 128, 128), **x)
        runs.append((out, st.dev))
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(r, runs[0]))


def test_slots_past_four_gib(ctx):
    k = kvx()
    heads, p, n = 1, 64, 64
    slot_bytes = 1 << 20
    pool = torch.zeros((5 << 30,), dtype=torch.uint8, device="cuda")
    count = pool.numel() // slot_bytes
    slots = k.StateSlots(pool, count, slot_bytes, recurrent_offset=4096)
    for lens, single in (([1], True), ([100], False)):
        data = Inputs(lens[0], heads, p, n, 1, BF16)
        batch, _ = batch_of(lens, [count - 2], [count - 1], single=single)
        out = torch.empty((lens[0], heads, p), dtype=BF16, device="cuda")
        k.kv_state_delta(ctx, slots, batch, out=out, A=data.A.cuda(), workspace=k.kv_state_delta_workspace(ctx, batch, heads, p, n), **data.cuda())
        after = pool.view(count, slot_bytes)[-1, 4096:4096 + p * n * 4].view(torch.float32).view(heads, p, n).cpu().double()
        c = data.cpu()
        y, state, slack, terms, q = mixers.delta(c["query"], c["key"], c["value"], c["beta"], torch.zeros((heads, p, n)), c["dt"], data.A)
        close(out.cpu().double(), y, after, state, slack, terms, q, BF16, True)


def test_an_output_over_an_input_is_refused(ctx):
    k = kvx()
    st = Slots(2, 2, 64, 64)
    for lens in ([100, 3], [1, 1]):
        batch, starts = batch_of(lens, [0, 1])
        data = Inputs(starts[-1], 2, 64, 64, 2, BF16)
        x = data.cuda()
        before = {name: v.clone() for name, v in x.items()}
        ws = k.kv_state_delta_workspace(ctx, batch, 2, 64, 64)
        for name in ("query", "key", "value"):
            with pytest.raises(k.KvxError) as e:
                k.kv_state_delta(ctx, st.slots, batch, out=x[name], A=data.A.cuda(), workspace=ws, **x)
            assert e.value.status == k.KVX_EINVAL
        torch.cuda.synchronize()
        assert all(torch.equal(x[name], before[name]) for name in before) and torch.equal(st.dev.cpu(), st.cpu)


def test_refusals(ctx):
    """Each returns its status before anything is enqueued and leaves the outputs alone."""
    k = kvx()
    st = Slots(2, 2, 64, 64)
    batch, _ = batch_of([100, 3], [0, 1])
    data = Inputs(103, 2, 64, 64, 1, BF16)
    x, A = data.cuda(), data.A.cuda()
    out = torch.full((103, 2, 64), 7.0, dtype=BF16, device="cuda")
    ws = k.kv_state_delta_workspace(ctx, batch, 2, 64, 64)

    def call(status, slots=st.slots, batch=batch, ws=ws, out=out, A=A, options={}, **other):
        with pytest.raises(k.KvxError) as e:
            k.kv_state_delta(ctx, slots, batch, out=out, A=A, workspace=ws, **{**x, **other}, **options)
        assert e.value.status == status, e.value

    call(k.KVX_EINVAL, options={"scale": math.inf})
    call(k.KVX_EINVAL, options={"eps": -1.0})
    call(k.KVX_EINVAL, query=x["query"][..., :48], key=x["key"][..., :48])
    three = torch.zeros((103, 3, 64), dtype=BF16, device="cuda")
    call(k.KVX_EINVAL, query=three, key=three)
    call(k.KVX_EALIGN, value=x["value"][..., :60], out=out[..., :60])
    call(k.KVX_EALIGN, value=torch.zeros((103, 2, 72), dtype=BF16, device="cuda")[..., 4:68])
    call(k.KVX_EINVAL, out=torch.zeros((103, 1, 64), dtype=BF16, device="cuda").expand(103, 2, 64))
    call(k.KVX_EDEVICE, out=out.cpu())
    call(k.KVX_EDEVICE, beta=x["beta"].cpu())
    call(k.KVX_EDEVICE, A=A.cpu())
    call(k.KVX_ERANGE, slots=k.StateSlots(st.dev, 2, st.bytes, recurrent_offset=1024))
    if ws.numel() > 16:
        call(k.KVX_ERANGE, ws=ws[:16])
        call(k.KVX_ERANGE, ws=None)
        call(k.KVX_EALIGN, ws=torch.zeros(ws.numel() + 16, dtype=torch.uint8, device="cuda")[4:])
    for bad in ({"query": x["query"][:5]}, {"beta": x["beta"][:, :1]}, {"dt": x["dt"][:5]}, {"scale": 0.0}):
        with pytest.raises(ValueError):
            k.kv_state_delta(ctx, st.slots, batch, out=out, A=A, workspace=ws, **{**x, **bad})
    with pytest.raises(ValueError):
        k.kv_state_delta(ctx, st.slots, batch, out=out, workspace=ws, **x)
    with pytest.raises(TypeError):
        k.kv_state_delta(ctx, st.slots, batch, out=out.half(), A=A, workspace=ws, **x)
    k.kv_fault_inject("launch")
    call(k.KVX_ECUDA)
    torch.cuda.synchronize()
    assert bool((out == 7.0).all()) and torch.equal(st.dev.cpu(), st.cpu)
    empty = k.StateBatch(torch.zeros(0, dtype=torch.int32, device="cuda"), starts=ints([0]), tokens=0)
    before = k.kv_ctx_stats(ctx)["kernel_launches"]
    none = {name: v[:0] for name, v in x.items()}
    k.kv_state_delta(ctx, st.slots, empty, out=out[:0], A=A, **none)
    assert k.kv_ctx_stats(ctx)["kernel_launches"] == before


def test_mixers_of_a_hybrid_models_steps(ctx):
    """A prompt, then single tokens and a draft of three through an attention layer over picked pages and a gated delta layer, each
    step against the plain forms on what the steps before left."""
    k = kvx()
    heads, hq, d, block, budget = 2, 8, 64, 16, 6
    lengths = [0, 0]
    tables, blocks = refs.tables_for([400, 200], block, 41)
    pages = refs.Pages(1, blocks, heads, block, d, BF16, seed=42)
    layer = pages.data[0].cuda()
    pool = k.KvPool.from_tensors([layer], heads, block)
    on_device = ints(lengths)
    batch = k.KvBatch(tables.cuda(), on_device, max_length=400)
    bounds = k.KvBounds.for_pool(pool)
    freq = (10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)).float()
    weights = [normal((d,), BF16, 43 + i, 0.1) + 1 for i in range(2)]
    rotary = k.KvRotary(hq, freq.cuda(), q_weight=weights[0].cuda(), k_weight=weights[1].cuda())
    st = Slots(2, hq, d, 64)
    state = [torch.zeros((hq, d, 64), dtype=torch.float64) for _ in range(2)]
    slack = [torch.zeros((hq, d), dtype=torch.float64) for _ in range(2)]
    for step, new in enumerate([[330, 150], [1, 1], [3, 3], [1, 1]]):
        lengths = [a + b for a, b in zip(lengths, new)]
        on_device.copy_(ints(lengths))
        t, starts = sum(new), [0, new[0], sum(new)]
        qkv = normal((t, hq + 2 * heads, d), BF16, 50 + step)
        dev = qkv.cuda()
        k.kv_append_rotary(ctx, pool, 0, batch, rotary, dev[:, :hq], dev[:, hq:hq + heads], dev[:, hq + heads:], dev[:, :hq], starts=ints(starts))
        k.kv_bounds(ctx, pool, 0, batch, bounds, new_tokens=max(new))
        q = dev[:, :hq]
        if new[0] == new[1]:
            n = new[0]
            sel, att = k.KvSelection(hq, budget, sinks=1, recent=2, new_tokens=n), k.KvAttention(hq, new_tokens=n)
            picked = torch.empty((t, heads, budget), dtype=torch.int32, device="cuda")
            out = torch.empty((t, hq, d), dtype=BF16, device="cuda")
            k.kv_select(ctx, pool, batch, bounds, sel, q, picked, k.kv_select_workspace(ctx, pool, batch, sel))
            k.kv_attend_selected(ctx, pool, 0, batch, att, picked, q, out, k.kv_attend_selected_workspace(ctx, pool, batch, att, budget))
            torch.cuda.synchronize()
            pages.data = layer.cpu()[None]
            rows, on_host = q.cpu(), picked.cpu()
            for s in range(2):
                made = [mixers.bounds_of(mixers.keys_of(pages, 0, tables[s], p, min(block, lengths[s] - p * block))) for p in range(-(-lengths[s] // block))]
                boxes, sizes = torch.stack([m[0] for m in made]), torch.stack([m[1] for m in made])
                for i in range(n):
                    score = mixers.scores_of(rows[s * n + i], boxes, sizes, heads)
                    count = (lengths[s] - n + i) // block + 1
                    assert [on_host[s * n + i, h].tolist() for h in range(heads)] == [mixers.pick(score[h], count, budget, 1, 2) for h in range(heads)]
            want, _, bound, _ = mixers.attend_selected(pages, 0, tables, lengths, rows, n, on_host, 1 / 8)
            assert bool(((out.cpu().double() - want).abs() <= bound).all())
        at = [lengths[s] - new[s] + i for s in range(2) for i in range(new[s])]
        want, size = mixers.rotate(qkv[:, :hq], at, freq, False, 1.0, weights[0], 1e-6, 0.0)
        assert bool(((q.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18 * size).all())
        data = Inputs(t, hq, d, 64, 4, BF16, seed=60 + step)
        batch_s = k.StateBatch(ints([1, 0]), starts=ints(starts), tokens=t, fresh=ints([step == 0] * 2))
        y = torch.empty((t, hq, d), dtype=BF16, device="cuda")
        k.kv_state_delta(ctx, st.slots, batch_s, out=y, A=data.A.cuda(), dt_bias=data.bias.cuda(),
                         workspace=k.kv_state_delta_workspace(ctx, batch_s, hq, d, 64), **data.cuda())
        torch.cuda.synchronize()
        c = data.cpu()
        after = st.dev.cpu()[:, :st.rec].view(torch.float32).view(2, hq, d, 64).double()
        for s in range(2):
            rows = slice(starts[s], starts[s + 1])
            want, state[s], more, terms, q64 = mixers.delta(c["query"][rows], c["key"][rows], c["value"][rows], c["beta"][rows], state[s],
                                                            c["dt"][rows], data.A, data.bias)
            # what the steps before were off by is carried along, and fades with the state
            close(y[rows].cpu().double(), want, after[1 - s], state[s], more + slack[s], terms, q64, BF16, True)
            slack[s] = slack[s] + more[-1]
    assert k.kv_get_device_error(ctx) == -1
