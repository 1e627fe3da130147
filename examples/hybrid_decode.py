"""A hybrid model's layers computed on the pages and state slots that the tier moves (paper Sec. 2.2).

Replica A takes a 2,048-token prompt through the token mixers of a 64-layer hybrid (16 attention layers of 8 KV
heads x 128 dims, bf16, 16-token pages; 48 recurrent layers of 16 heads x 128 x 128): new K/V into the pages, attention
of the prompt's last 64 tokens that accumulates how much each cached token is used, the short convolution and the
selective scan on the state slots.  It then keeps the 512 tokens that were used most in every layer and head, stores
their pages and the state snapshot in pinned host memory, and replica B restores both into pages and slots of its own.
Both go on with the same eight tokens.  Projections and everything between the layers are random numbers, the same for
both; at every token B's outputs must be A's, bit for bit, whatever the pages they came from.

Run from the repository root, with the library built:
    python examples/hybrid_decode.py
Prints the times of each part and "decode bit-exact" and exits 0 on success.
"""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

PROMPT, WINDOW, KEEP, DECODE = 2048, 64, 512, 8
Q_HEADS, STATE_HEADS, STATE_DIM, GROUPS, CHANNELS, WIDTH = 32, 16, 128, 8, 8192, 4
BF16 = torch.bfloat16


def numbers(shape, seed, scale=1.0, dtype=BF16):
    """What the model's projections would have put out."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


class Layers:
    """One replica's pages, tables and slots, and the layers' weights (the same on every replica)."""

    def __init__(self, k, shape, ctx, pages, seed):
        self.k, self.shape, self.ctx = k, shape, ctx
        self.pages = [torch.zeros((pages, 2, shape.kv_heads, shape.block_tokens, shape.head_dim), dtype=BF16, device="cuda")
                      for _ in range(shape.attn_layers)]
        self.pool = k.KvPool.from_tensors(self.pages, shape.kv_heads, shape.block_tokens)
        self.free = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32).cuda()
        self.taken = 0
        self.state = [torch.zeros(shape.state_bytes, dtype=torch.uint8, device="cuda") for _ in range(shape.state_layers)]
        self.slots = [k.StateSlots(s, 1, shape.state_bytes, 0, shape.recurrent_bytes) for s in self.state]
        self.slot = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.length = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.conv_weight = numbers((CHANNELS, WIDTH), 1, 0.5)
        self.A = -torch.exp(numbers((STATE_HEADS,), 2, 1.0, torch.float32))
        self.D = numbers((STATE_HEADS,), 3, 1.0, torch.float32)
        self.dt_bias = numbers((STATE_HEADS,), 4, 1.0, torch.float32) - 4.0

    def take(self, tokens):
        """A table of fresh pages for so many tokens."""
        n = -(-tokens // self.shape.block_tokens)
        self.taken += n
        return self.free[None, self.taken - n:self.taken].contiguous()

    def use(self, table, tokens):
        self.table, self.batch = table, self.k.KvBatch(table, self.length)
        self.length.fill_(tokens)
        self.attention = {n: self.k.KvAttention(Q_HEADS, new_tokens=n) for n in (1, WINDOW)}
        self.workspace = {n: self.k.kv_attend_workspace(self.ctx, self.pool, self.batch, a, weights=n > 1)
                          for n, a in self.attention.items()}

    def attend(self, layer, seed, new, queries, weights=None):
        """An attention layer over `new` tokens, the last `queries` of which attend."""
        s, k = self.shape, self.k
        qkv = numbers((new, Q_HEADS + 2 * s.kv_heads, s.head_dim), seed)
        k.kv_append(self.ctx, self.pool, layer, self.batch, qkv[:, Q_HEADS:Q_HEADS + s.kv_heads],
                    qkv[:, Q_HEADS + s.kv_heads:], new_tokens=new)
        out = torch.empty((queries, Q_HEADS, s.head_dim), dtype=BF16, device="cuda")
        k.kv_attend(self.ctx, self.pool, layer, self.batch, self.attention[queries], qkv[new - queries:, :Q_HEADS], out,
                    self.workspace[queries], weights=weights)
        return out

    def recur(self, layer, seed, new, fresh=False):
        """A recurrent layer over `new` tokens: its convolution, and the scan of what it puts out."""
        k, h, n = self.k, STATE_HEADS, STATE_DIM
        starts = torch.tensor([0, new], dtype=torch.int32, device="cuda") if new > 1 else None
        batch = k.StateBatch(self.slot, starts=starts, tokens=new,
                             fresh=torch.ones(1, dtype=torch.int32, device="cuda") if fresh else None)
        x = numbers((new, CHANNELS), seed, 0.5)
        mixed = torch.empty_like(x)
        k.kv_state_conv(self.ctx, self.slots[layer], batch, x, self.conv_weight, mixed)
        out = torch.empty((new, h, n), dtype=BF16, device="cuda")
        at, size = h * n, GROUPS * n
        k.kv_state_scan(self.ctx, self.slots[layer], batch, mixed[:, :at].view(new, h, n), numbers((new, h), seed + 1), self.A,
                        mixed[:, at:at + size].view(new, GROUPS, n), mixed[:, at + size:at + 2 * size].view(new, GROUPS, n), out,
                        D=self.D, dt_bias=self.dt_bias, workspace=k.kv_state_scan_workspace(self.ctx, batch, h, n, n))
        return out


def main():
    from paper_2609_15021_gb300 import kvxfer as k
    from paper_2609_15021_gb300.hybrid import HybridShape
    shape = HybridShape()
    ctx = k.kv_ctx_create(0)
    host = k.HostBuffer(KEEP // shape.chunk_tokens * shape.chunk_bytes)
    snapshot = k.HostBuffer(shape.snapshot_bytes)
    chunks = [host.tensor[i * shape.chunk_bytes:(i + 1) * shape.chunk_bytes] for i in range(KEEP // shape.chunk_tokens)]
    try:
        a, b = Layers(k, shape, ctx, 256, 7), Layers(k, shape, ctx, 96, 8)
        parts = []

        def timed(name, f):
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            got = f()
            end.record()
            parts.append((name, begin, end))
            return got

        # A: the prompt
        a.use(a.take(PROMPT), PROMPT)
        weights = torch.zeros((shape.attn_layers, 1, shape.kv_heads, PROMPT), device="cuda")
        timed("prompt: attention layers", lambda: [a.attend(l, 1000 + l, PROMPT, WINDOW, weights[l]) for l in range(shape.attn_layers)])
        timed("prompt: recurrent layers", lambda: [a.recur(l, 3000 + 2 * l, PROMPT, fresh=True) for l in range(shape.state_layers)])
        # A: what attention used most, and room for what comes
        table = a.take(KEEP + DECODE)
        kept = torch.empty((shape.attn_layers, 1, shape.kv_heads, KEEP), dtype=torch.int32, device="cuda")
        length = torch.empty(1, dtype=torch.int32, device="cuda")
        timed("eviction", lambda: k.kv_evict(ctx, a.pool, a.batch, weights, KEEP, table, kept, length, sinks=4, recent=WINDOW))
        a.use(table, KEEP)

        def store():
            k.kv_store(ctx, a.pool, table, 0, KEEP, shape.chunk_tokens, chunks)
            k.kv_state_store(ctx, a.state, 1, shape.state_bytes, 0, snapshot.tensor)

        def restore():
            k.kv_load(ctx, b.pool, b.table, 0, KEEP, shape.chunk_tokens, chunks)
            k.kv_state_load(ctx, b.state, 1, shape.state_bytes, 0, snapshot.tensor)

        timed("store", store)
        b.use(b.take(KEEP + DECODE), KEEP)
        timed("restore", restore)
        for token in range(DECODE):
            outs = []
            for r in (a, b):
                r.length.add_(1)
                seed = 100000 * (token + 1)
                outs.append([r.attend(l, seed + l, 1, 1) for l in range(shape.attn_layers)] +
                            [r.recur(l, seed + 1000 + 2 * l, 1) for l in range(shape.state_layers)])
            if not all(torch.equal(x, y) for x, y in zip(*outs)):
                raise SystemExit(f"token {token}: the replicas' outputs differ")
            if not all(bool(torch.isfinite(x).all()) for x in outs[0]):
                raise SystemExit(f"token {token}: outputs are not finite")
        torch.cuda.synchronize()
        if int(length) != KEEP or not bool((kept[..., 1:] > kept[..., :-1]).all()):
            raise SystemExit("the eviction did not keep what it should")
        if k.kv_get_device_error(ctx) != -1:
            raise SystemExit("a block-table entry, a length or a slot was out of range")
        for name, begin, end in parts:
            print(f"{name}: {begin.elapsed_time(end):.2f} ms")
        print(f"{PROMPT} tokens shrunk to {KEEP} and moved; {DECODE} tokens on both replicas: decode bit-exact")
    finally:
        k.kv_ctx_destroy(ctx)
        host.close()
        snapshot.close()


if __name__ == "__main__":
    main()
