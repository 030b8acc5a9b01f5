"""A language model's attention block at 8 and 4 bits, on the library's calls.

    x --int8 product--> q, k, v --rotation--> cache (4 bits) --attention--> int8 product --> y

A batch of sequences of different lengths is processed as prompts, then decoded
token by token; the cache is paged and grows a page at a time.  Run as a script,
it compares the block with the same block on unquantized weights and an
unquantized cache, and times a decoding step replayed from a graph:

    python examples/attention_block.py
"""
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1705_01462_amd as fgq  # noqa: E402


def rotate(x, pos):
    """Rotary positions of x [tokens][heads][D] (halves form the pairs)."""
    half = x.shape[-1] // 2
    freq = 10000.0 ** (-torch.arange(half, device=x.device, dtype=torch.float32) / half)
    angle = pos.to(torch.float32)[:, None, None] * freq
    a, b = x.float().chunk(2, -1)
    c, s = angle.cos(), angle.sin()
    return torch.cat((a * c - b * s, a * s + b * c), -1).to(x.dtype)


class Pages:
    """Which pages of the cache a batch of sequences owns."""

    def __init__(self, num_pages, batch, max_tokens, P, device="cuda"):
        self.P, self.free = P, list(range(num_pages))
        self.table = torch.zeros((batch, -(-max_tokens // P)), dtype=torch.int32, device=device)
        self.lens = [0] * batch

    def extend(self, counts):
        """Make room for counts[b] more tokens of each sequence; returns their slots (int64)."""
        slots = []
        for b, n in enumerate(counts):
            for t in range(self.lens[b], self.lens[b] + n):
                if t % self.P == 0:
                    self.table[b, t // self.P] = self.free.pop()
            self.lens[b] += n
        owned = self.table.tolist()
        for b, n in enumerate(counts):
            slots += [owned[b][t // self.P] * self.P + t % self.P for t in range(self.lens[b] - n, self.lens[b])]
        return torch.tensor(slots, dtype=torch.int64, device=self.table.device)


class AttentionBlock:
    """Weights wqkv [(Hq + 2 Hkv) D][E] and wo [E][Hq D] (any float type), kept as
    int8 rows with a scale each; a cache of `bits` bits in groups of G channels."""

    def __init__(self, wqkv, wo, Hq, Hkv, D, num_pages, P=16, bits=4, G=64):
        self.Hq, self.Hkv, self.D, self.P, self.bits, self.G = Hq, Hkv, D, P, bits, G
        self.wqkv, self.sqkv = fgq.fgq_quantize_rows(wqkv)
        self.wo, self.so = fgq.fgq_quantize_rows(wo)
        self.cache = fgq.fgq_kv_cache(num_pages, Hkv, D, P, bits, G, device=wqkv.device)

    def attend(self, x, pos, slots, cu_q, max_q, pages, kv_lens, window=0):
        """Attention of the tokens x [T][E] (float16 or bfloat16) at positions pos,
        their keys and values written to the cache's slots first: [T][Hq D]."""
        qkv = fgq.fgq_linear_i8(x, self.wqkv, self.sqkv)
        qkv = qkv.unflatten(1, (self.Hq + 2 * self.Hkv, self.D))
        q = rotate(qkv[:, :self.Hq], pos)
        k = rotate(qkv[:, self.Hq:self.Hq + self.Hkv], pos)
        fgq.fgq_kv_write(k, qkv[:, self.Hq + self.Hkv:], slots, self.cache, self.P, self.bits, self.G)
        o = fgq.fgq_attn_kv(q, cu_q, max_q, self.cache, pages, kv_lens, self.P, self.bits, self.G, window=window)
        return o.flatten(1)

    def __call__(self, *args, **kw):
        return fgq.fgq_linear_i8(self.attend(*args, **kw), self.wo, self.so)


def batch(counts, lens, device="cuda"):
    """cu_q, max_q, positions and key counts of counts[b] new tokens behind lens[b] - counts[b] earlier ones."""
    cu = [0]
    pos = []
    for n, total in zip(counts, lens):
        cu.append(cu[-1] + n)
        pos += range(total - n, total)
    i32 = dict(dtype=torch.int32, device=device)
    return torch.tensor(cu, **i32), max(counts), torch.tensor(pos, **i32), torch.tensor(lens, **i32)


def plain(x, wqkv, wo, Hq, Hkv, D, counts):
    """The block in fp32 on unquantized weights, whole sequences at once."""
    qkv = (x.float() @ wqkv.float().t()).unflatten(1, (Hq + 2 * Hkv, D))
    out, at = [], 0
    for n in counts:
        pos = torch.arange(n, device=x.device)
        s = qkv[at:at + n]
        at += n
        q, k, v = rotate(s[:, :Hq], pos), rotate(s[:, Hq:Hq + Hkv], pos), s[:, Hq + Hkv:]
        k, v = (t.repeat_interleave(Hq // Hkv, 1).transpose(0, 1).contiguous() for t in (k, v))
        sc = q.transpose(0, 1).contiguous() @ k.transpose(1, 2).contiguous() * D ** -0.5
        sc = sc.masked_fill(torch.triu(torch.ones_like(sc[0], dtype=torch.bool), 1), float("-inf"))
        out.append((sc.softmax(-1) @ v).transpose(0, 1).flatten(1))
    return torch.cat(out) @ wo.float().t()


def main():
    Hq, Hkv, D, E, P, steps = 16, 4, 128, 2048, 16, 64
    prompts = [700, 33, 410, 256]
    g = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    wqkv, wo = rnd((Hq + 2 * Hkv) * D, E) / E ** 0.5, rnd(E, Hq * D) / (Hq * D) ** 0.5
    total = [n + steps for n in prompts]
    x = [rnd(n, E).to(torch.bfloat16) for n in total]
    num_pages = sum(-(-n // P) for n in total)
    block = AttentionBlock(wqkv, wo, Hq, Hkv, D, num_pages, P)
    pages = Pages(num_pages, len(prompts), max(total), P)

    # the prompts
    slots = pages.extend(prompts)
    cu, mq, pos, lens = batch(prompts, pages.lens)
    y = block(torch.cat([t[:n] for t, n in zip(x, prompts)]), pos, slots, cu, mq, pages.table, lens)
    got = [list(t.split(1)) for t in y.split(prompts)]

    # token by token: inputs of a step in place, the step itself a graph
    one = [1] * len(prompts)
    cu, mq, pos, lens = batch(one, [n + 1 for n in prompts])
    slots = torch.full((len(prompts),), -1, dtype=torch.int64, device="cuda")
    xs = torch.zeros(len(prompts), E, dtype=torch.bfloat16, device="cuda")
    table = pages.table.clone()
    block(xs, pos, slots, cu, mq, table, lens)  # once outside the graph (slots -1: nothing is written)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ys = block(xs, pos, slots, cu, mq, table, lens)
    for s in range(steps):
        new = pages.extend(one)
        slots.copy_(new)
        table.copy_(pages.table)
        lens.copy_(torch.tensor(pages.lens, dtype=torch.int32))
        pos.copy_(torch.tensor([n - 1 for n in pages.lens], dtype=torch.int32))
        xs.copy_(torch.stack([t[n + s] for t, n in zip(x, prompts)]))
        graph.replay()
        for b, row in enumerate(ys.clone().split(1)):
            got[b].append(row)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(200):
        graph.replay()
    torch.cuda.synchronize()
    us = (time.perf_counter() - t) / 200 * 1e6

    want = plain(torch.cat(x), wqkv, wo, Hq, Hkv, D, total)
    have = torch.cat([torch.cat(r) for r in got]).float()
    err = ((have - want).norm() / want.norm()).item()
    print(f"{len(prompts)} sequences, {sum(prompts)} prompt tokens and {steps} steps: relative difference to the "
          f"unquantized block {err:.3f}; {us:.1f} us a decoding step")
    return err


if __name__ == "__main__":
    main()
