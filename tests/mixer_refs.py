"""Plain 64-bit statements of the rotated append, the bounds and choice of pages, attention over chosen pages and the gated
delta rule, on the CPU, with what the tests' error bounds are made of."""
from __future__ import annotations

import math

import torch

from operator_refs import UNIT


def rotate(x, positions, inv_freq, interleaved, scale, weight, eps, offset):
    """(rows, sizes) of x [T][H][D]: normed and rotated rows in 64 bits, and the sum of absolute values of the terms that
    each element is the sum of."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * (weight.double() + offset)
    out, size = x.clone(), x.abs()
    half = 0 if inv_freq is None else inv_freq.shape[0]
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        for t, p in enumerate(positions):
            angle = math.remainder(p * float(inv_freq[i]), 2 * math.pi)
            c, s = math.cos(angle) * scale, math.sin(angle) * scale
            out[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            out[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
            size[t, :, a] = size[t, :, b] = (x[t, :, a].abs() + x[t, :, b].abs()) * abs(scale)
    return out, size


def keys_of(pages, layer, table, page, tokens):
    """Keys [token][head][dim] of the first `tokens` tokens of a sequence's page."""
    return pages.rows(layer, table, range(page * pages.block, page * pages.block + tokens))[0]


def bounds_of(keys):
    """(box [head][2][dim] int8, size [head] float32) of keys [token][head][dim], in 32 bits as stored."""
    k = keys.float()
    low, high = k.amin(0), k.amax(0)
    odd = ~torch.isfinite(k).all(0).all(-1)
    size = torch.maximum(low.abs(), high.abs()).amax(-1) / torch.tensor(127.0)
    by = torch.where(size > 0, size, torch.tensor(1.0))[:, None]
    box = torch.stack([torch.floor(low / by), torch.ceil(high / by)], 1).clamp(-127, 127)
    box[odd, 0], box[odd, 1] = -127.0, 127.0
    return box.to(torch.int8), torch.where(odd, torch.tensor(torch.finfo(torch.float32).max), size)


def scores_of(q, boxes, sizes, heads):
    """Scores [head][page] in 32 bits of one query q [Hq][D] by boxes [page][head][2][dim] and sizes [page][head]."""
    group = q.shape[0] // heads
    q = q.float()
    top = q.abs().amax(-1, keepdim=True)
    fine = torch.isfinite(q).all(-1, keepdim=True)
    step = torch.where(fine, top / torch.tensor(127.0), torch.tensor(0.0))
    whole = torch.where(step > 0, torch.round(q / torch.where(step > 0, step, torch.tensor(1.0))), torch.tensor(0.0))
    whole = whole.clamp(-127, 127).long()
    out = torch.empty((heads, boxes.shape[0]))
    for h in range(heads):
        w, low, high = whole[h * group:(h + 1) * group, None], boxes[:, h, 0].long(), boxes[:, h, 1].long()
        dots = (w.clamp(min=0) * high + w.clamp(max=0) * low).sum(-1)  # [row][page]
        out[h] = (dots.float() * step[h * group:(h + 1) * group]).amax(0) * sizes[:, h]
    return out


def pick(scores, pages, budget, sinks, recent):
    """Picked pages of one query and head, by a sort of (score, page)."""
    if pages <= budget:
        return list(range(pages))
    always = set(range(min(sinks, pages))) | set(range(max(0, pages - recent), pages))
    value = {j: -math.inf if math.isnan(scores[j]) else float(scores[j]) for j in range(pages) if j not in always}
    return sorted(always | set(sorted(value, key=lambda j: (-value[j], j))[:budget - len(always)]))


def attend_selected(pages, layer, tables, lengths, q, new, selected, scale, softcap=0.0, k_scale=1.0, v_scale=1.0,
                    missing=()):
    """(out, lse, bound on |out - exact|, bound on a probability's relative error): attention of the last `new` tokens over
    the tokens of selected pages [S * new][H][budget], with the bounds of attention over all keys."""
    hq, d = q.shape[1], q.shape[2]
    group = hq // pages.heads
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    bound = torch.zeros(q.shape, dtype=torch.float64)
    worst = 0.0
    unit_p = UNIT.get(pages.dtype, 2.0 ** -11)
    for s, n in enumerate(lengths):
        for t in range(new):
            pos = n - new + t
            for h in range(pages.heads):
                seen, before = [], -1
                for page in selected[s * new + t, h].tolist():
                    if page > before and page * pages.block <= pos and (s, page // pages.pack) not in missing:
                        seen += [j for j in range(page * pages.block, (page + 1) * pages.block) if j <= pos]
                    before = page
                if not seen or pos < 0:
                    continue
                kv = pages.rows(layer, tables[s], seen)[:, :, h].double()
                k, v = kv[0] * k_scale, kv[1] * v_scale
                for i in range(h * group, (h + 1) * group):
                    row = q[s * new + t, i].double()
                    score = (k @ row) * scale
                    amp = float((k.abs() @ row.abs()).max()) * abs(scale)
                    if softcap:
                        score = softcap * torch.tanh(score / softcap)
                    l = torch.logsumexp(score, 0)
                    p = torch.exp(score - l)
                    err = 2 * d * 2.0 ** -24 * amp + 2.0 ** -16 + softcap * 2.0 ** -20
                    worst = max(worst, err)
                    out[s * new + t, i] = p @ v
                    lse[s * new + t, i] = l
                    bound[s * new + t, i] = UNIT[q.dtype] * (p @ v).abs() + (unit_p + err) * (p @ v.abs()) + 1e-7
    return out, lse, bound, worst


def delta(q, k, v, beta, state, dt=None, A=None, dt_bias=None, softplus=True, sigmoid=True, normalize=True, eps=1e-6,
          scale=None):
    """(out, state, slack, terms) of one sequence in 64 bits, token by token: q, k [T][G][N], v [T][H][P], beta, dt [T][H],
    state [H][P][N].

    slack [T + 1][H][P]: sums of the sizes of what each step adds up for a row of the state, carried with the decay: a
    rounding error of u in every step's numbers is one of the row (as a vector) of at most u times this, as a step
    s -> a (s - b (s.k) k) does not lengthen a vector where b |k|^2 <= 2.  slack[t] is before token t, the last one
    after all.  terms [T][H][P]: sum over s <= t of |q_t . k_s| decay |d_s|, the terms of the output's product form."""
    t_n, h = v.shape[:2]
    per = h // k.shape[1]
    n = k.shape[-1]
    scale = 1 / math.sqrt(n) if scale is None else scale
    q, k, v, beta = (x.double() for x in (q, k, v, beta))
    if normalize:
        q, k = (x / torch.sqrt((x * x).sum(-1, keepdim=True) + eps) for x in (q, k))
    q, k = (q * scale).repeat_interleave(per, 1), k.repeat_interleave(per, 1)
    beta = 1 / (1 + torch.exp(-beta)) if sigmoid else beta
    state = state.double().clone()
    rows, slack, size, terms = [], [], torch.zeros(state.shape[:2], dtype=torch.float64), []
    wrote = torch.zeros((0, h, v.shape[2]), dtype=torch.float64)
    faded = torch.zeros((0, h), dtype=torch.float64)
    for t in range(t_n):
        a = torch.ones(h, dtype=torch.float64)
        if dt is not None:
            d = dt[t].double() + (0 if dt_bias is None else dt_bias.double())
            d = torch.nn.functional.softplus(d, threshold=1e9) if softplus else d
            a = torch.exp(d * A.double())
        slack.append(size)
        state = state * a[:, None, None]
        held = (state * k[t][:, None, :]).sum(-1)
        write = beta[t][:, None] * (v[t] - held)
        norm = torch.linalg.vector_norm(k[t], dim=-1)[:, None]
        length = torch.linalg.vector_norm(state, dim=-1)
        size = size * a[:, None] + length + beta[t].abs()[:, None] * norm * (v[t].abs() + 2 * length * norm)
        state = state + write[:, :, None] * k[t][:, None, :]
        rows.append((state * q[t][:, None, :]).sum(-1))
        wrote, faded = torch.cat([wrote, write.abs()[None]]), torch.cat([faded * a, torch.ones((1, h), dtype=torch.float64)])
        terms.append((((k[:t + 1] * q[t]).sum(-1).abs() * faded)[..., None] * wrote).sum(0))
    slack.append(size)
    empty = v.clone()
    return (torch.stack(rows) if rows else empty), state, torch.stack(slack), (torch.stack(terms) if terms else empty), q
