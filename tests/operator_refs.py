"""Plain 64-bit statements of the operators on pages and state slots, on the CPU and token by
token, with the sums of absolute values that the tests' error bounds are made of."""
from __future__ import annotations

import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # rounding to the type: 8 and 11 significant bits
E4M3_MAX = 448.0


class Pages:
    """A one-layer (or more) pool on the CPU with its tables: pages [layer][page][2][H][B][D] or [..][2][B][H][D]."""

    def __init__(self, layers, blocks, heads, block, dim, dtype, nhd=False, pack=1, seed=0, fill=None):
        self.heads, self.block, self.dim, self.dtype, self.nhd, self.pack = heads, block, dim, dtype, nhd, pack
        shape = (layers, blocks * pack, 2, block, heads, dim) if nhd else (layers, blocks * pack, 2, heads, block, dim)
        g = torch.Generator().manual_seed(seed)
        self.data = (torch.randn(shape, generator=g) if fill is None else torch.full(shape, fill)).to(dtype)

    def rows(self, layer, table, positions):
        """K and V rows [2][position][head][dim] (a view's copy) of the positions, as stored."""
        out = []
        for p in positions:
            page = int(table[p // self.block // self.pack]) * self.pack + p // self.block % self.pack
            half = self.data[layer, page]
            out.append(half[:, p % self.block] if self.nhd else half[:, :, p % self.block])
        return torch.stack(out, 1) if out else self.data.new_zeros((2, 0, self.heads, self.dim))

    def put(self, layer, table, p, rows):
        """rows [2][head][dim], already of the pool's type."""
        page = int(table[p // self.block // self.pack]) * self.pack + p // self.block % self.pack
        if self.nhd:
            self.data[layer, page, :, p % self.block] = rows
        else:
            self.data[layer, page, :, :, p % self.block] = rows


def quantise(x, scale):
    """As an e4m3 cache stores x: the quotient in 32 bits, clamped, rounded to nearest even."""
    return (x.float() / torch.tensor(scale, dtype=torch.float32)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def tables_for(lengths, span, seed, spare=1, bad=-1):
    """Block tables of randomly ordered pages, `bad` behind each sequence's last."""
    need = [-(-n // span) for n in lengths]
    total = sum(need) + spare
    order = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    tables = torch.full((len(lengths), max(need + [0]) + 1), bad, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        tables[s, :n] = order[at:at + n]
        at += n
    return tables, total


def attend(pages, layer, tables, lengths, q, new, scale, softcap=0.0, window=0, slopes=None, k_scale=1.0,
           v_scale=1.0, missing=()):
    """(out, lse, weights, bound on |out - exact|, bound on a probability's relative error) for
    q [S * new][Hq][D].  missing: logical blocks (sequence, block) whose table entries name no page.

    The bounds: a dot product of D terms in 32 bits is off by at most D * 2^-24 * sum |q k|; twice that (a
    probability and the sum it is divided by) and 2^-16 for exp and the sums is a probability's error; rounded to
    the cache's type (8-bit caches: fp16) in the product with V it is off by that type's unit more, and the result
    by its own type's."""
    hq, d = q.shape[1], q.shape[2]
    s_n, group = len(lengths), hq // pages.heads
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    bound = torch.zeros(q.shape, dtype=torch.float64)
    weights = torch.zeros((s_n, pages.heads, max(list(lengths) + [1])), dtype=torch.float64)
    unit_out = UNIT[q.dtype]
    unit_p = UNIT.get(pages.dtype, 2.0 ** -11)
    worst = 0.0
    for s, n in enumerate(lengths):
        for t in range(new):
            pos = n - new + t
            lo = max(0, pos + 1 - window) if window else 0
            span = pages.block * pages.pack
            seen = [j for j in range(lo, pos + 1) if (s, j // span) not in missing]
            if not seen:
                continue
            kv = pages.rows(layer, tables[s], seen).double()
            for i in range(hq):
                k, v = kv[0, :, i // group] * k_scale, kv[1, :, i // group] * v_scale
                row = q[s * new + t, i].double()
                score = (k @ row) * scale
                amp = float((k.abs() @ row.abs()).max()) * abs(scale)
                if softcap:
                    score = softcap * torch.tanh(score / softcap)
                if slopes is not None:
                    back = torch.tensor([j - pos for j in seen], dtype=torch.float64) * float(slopes[i])
                    score = score + back
                    amp += float(back.abs().max())
                l = torch.logsumexp(score, 0)
                p = torch.exp(score - l)
                err = 2 * d * 2.0 ** -24 * amp + 2.0 ** -16 + softcap * 2.0 ** -20
                worst = max(worst, err)
                out[s * new + t, i] = p @ v
                lse[s * new + t, i] = l
                bound[s * new + t, i] = unit_out * (p @ v).abs() + (unit_p + err) * (p @ v.abs()) + 1e-7
                weights[s, i // group, seen] += p
    return out, lse, weights, bound, worst


def select(weights, length, budget, sinks, recent):
    """Kept positions of one sequence and head, by a sort of (weight, position)."""
    keep = min(length, budget)
    if keep == length:
        return list(range(length))
    always = set(range(sinks)) | set(range(length - recent, length))
    value = {j: -math.inf if math.isnan(weights[j]) else float(weights[j]) for j in range(length) if j not in always}
    best = sorted(value, key=lambda j: (-value[j], j))[:keep - len(always)]
    return sorted(always | set(best))


def conv(x, weight, bias, window, silu):
    """(out, new window) of one sequence: x [T][C], weight [C][W], window [W-1][C], all float64."""
    w = weight.shape[1]
    full = torch.cat([window, x])
    out = []
    for t in range(x.shape[0]):
        y = (full[t:t + w] * weight.T).sum(0) + (0 if bias is None else bias)
        out.append(y / (1 + torch.exp(-y)) if silu else y)
    return (torch.stack(out) if out else x.clone()), full[x.shape[0]:]


def scan(x, dt, A, B, C, D, dt_bias, softplus, state):
    """(out, state, absolute out, absolute state) of one sequence, float64: x [T][H][P], dt [T][H], B, C [T][G][N].
    The absolute ones are the same recurrence over absolute values: the size of what was added up."""
    h = x.shape[1]
    per = h // B.shape[1]
    state, big = state.clone(), state.abs()
    out, size = [], []
    for t in range(x.shape[0]):
        d = dt[t] + (0 if dt_bias is None else dt_bias)
        d = torch.nn.functional.softplus(d, threshold=1e9) if softplus else d
        a = torch.exp(d * A)[:, None, None]
        b, c = B[t].repeat_interleave(per, 0), C[t].repeat_interleave(per, 0)
        add = (d[:, None] * x[t])[:, :, None] * b[:, None, :]
        state, big = state * a + add, big * a + add.abs()
        skip = 0 if D is None else D[:, None] * x[t]
        out.append((state * c[:, None, :]).sum(-1) + skip)
        size.append((big * c.abs()[:, None, :]).sum(-1) + (skip.abs() if D is not None else 0))
    empty = x.clone()
    return (torch.stack(out) if out else empty), state, (torch.stack(size) if size else empty), big
