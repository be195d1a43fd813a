"""A small streaming decoder on the paged pool: the operators and the swap used together, as a serving loop would.

Several requests share a system prompt, whose blocks they have in common.  Each step sets the batch once; every layer turns and
appends the new tokens' keys, attends (the prefix read once for all) and accumulates what each cached token was given.  A
request that has grown past its budget gives up its lightest tokens in all layers, and the blocks behind the rest go back to the
free list.  One request is preempted on the way: swapped out, its blocks handed to others, and swapped into different ones later.

The model is a stack of attention layers with random weights: there is nothing to learn from its tokens, only from how it runs.

    python -m paper_2510_02758_amd.stream_demo
"""
import numpy as np
import torch

from . import kvswap as kv
from . import workloads as W


class Stream:
    """The serving loop's state: tables, lengths, positions and accumulated weights of every request, and the pool they point into."""

    def __init__(self, device, n=3, budget=608, keep=560, seed=0):
        self.g = g = W.Geometry(L=4, H=2, D=64, B=16, dtype="bf16", N=128)
        self.n, self.G, self.budget, self.keep, self.device = n, 4, budget, keep, device
        self.Hq, self.width = g.H * self.G, 256
        gen = torch.Generator(device="cpu").manual_seed(seed)
        rand = lambda *s: (torch.randn(*s, generator=gen) * s[-1] ** -0.5).to(device, torch.bfloat16)  # noqa: E731
        self.qkv = [rand((self.Hq + 2 * g.H) * g.D, self.width) for _ in range(g.L)]
        self.proj = [rand(self.width, self.Hq * g.D) for _ in range(g.L)]
        rc, turns, self.magnitude = kv.kv_rope_freqs(g.D, 500000.0, kv.KV_ROPE_PARTS, factor=8.0, trained=8192.0)
        kv.kv_check(rc)
        self.turns = torch.from_numpy(turns).to(device)
        self.pool = torch.zeros(g.pool_bytes, dtype=torch.uint8, device=device)
        self.arena = torch.zeros(64 * g.S, dtype=torch.uint8, pin_memory=True)
        self.kp = kv.KVPool(g, self.pool, self.arena)
        self.batch = kv.KVBatch(self.kp)
        self.free = list(np.random.default_rng(seed).permutation(g.N))
        self.table, self.tokens, self.position = [[] for _ in range(n)], [0] * n, [0] * n
        self.cap = budget + 64
        self.weights = torch.zeros(g.L, n, g.H, self.cap, device=device)
        self.kept = torch.zeros(g.L, n, g.H, keep, dtype=torch.int32, device=device)
        self.evicted = 0

    def close(self):
        self.batch.close()
        self.kp.close()

    def _set(self, rows, new):
        """The batch of this step: `new[i]` tokens more for request rows[i]."""
        for i, k in zip(rows, new):
            self.tokens[i] += k
            self.position[i] += k
            while len(self.table[i]) * self.g.B < self.tokens[i]:
                self.table[i].append(self.free.pop())
        off = np.cumsum([0] + [len(self.table[i]) for i in rows]).astype(np.int32)
        ids = np.concatenate([self.table[i] for i in rows]).astype(np.int32)
        kv.kv_check(self.batch.set(off, ids, [self.tokens[i] for i in rows], new, self.Hq))
        return off, ids

    def step(self, rows, x, new):
        """Hidden states x [T, width] of the new tokens through all layers -> [T, width]."""
        g, T = self.g, x.shape[0]
        self._set(rows, new)
        where = np.concatenate([np.arange(self.position[i] - k, self.position[i]) for i, k in zip(rows, new)]).astype(np.int32)
        where = torch.from_numpy(where).to(self.device)
        # the batch's rows of the accumulators: all requests in order, or a copy of some
        some = self.weights if rows == list(range(self.n)) else self.weights[:, rows].contiguous()
        out = torch.empty(T, self.Hq, g.D, dtype=torch.bfloat16, device=self.device)
        for layer in range(g.L):
            qkv = (x @ self.qkv[layer].t()).view(T, self.Hq + 2 * g.H, g.D)
            q, k, v = qkv[:, :self.Hq], qkv[:, self.Hq:self.Hq + g.H], qkv[:, self.Hq + g.H:]
            kv.kv_check(self.batch.append(layer, q, k, v, turns=self.turns, magnitude=self.magnitude, positions=where))
            kv.kv_check(self.batch.attn(layer, q, out, g.D ** -0.5, weights=some[layer]))
            x = x + out.view(T, -1) @ self.proj[layer].t()
        if some is not self.weights:
            self.weights[:, rows] = some
        return x

    def evict(self, keep_first):
        """Requests past the budget go back to `keep` tokens; what lies behind these goes back to the free list."""
        crowded = [i for i in range(self.n) if self.tokens[i] > self.budget]
        if not crowded:
            return
        self._set(crowded, [0] * len(crowded))
        some = self.weights[:, crowded].contiguous()
        kept = self.kept[:, :len(crowded)].contiguous()
        kv.kv_check(self.batch.evict(0, self.g.L, some, kept, self.keep, keep_first=keep_first, keep_last=16, req_ids=crowded))
        self.weights[:, crowded] = some
        for i in crowded:
            self.evicted += self.tokens[i] - self.keep
            self.tokens[i] = self.keep
            blocks = -(-self.keep // self.g.B)
            self.free = self.table[i][blocks:] + self.free
            self.table[i] = self.table[i][:blocks]

    def preempt(self, i):
        torch.cuda.current_stream(self.device).synchronize()  # the swap runs on streams of its own
        kv.kv_check(self.kp.swap_out([i], [0, len(self.table[i])], np.array(self.table[i], np.int32), [self.tokens[i]]))
        kv.kv_check(self.kp.sync())

    def resume(self, i, blocks):
        kv.kv_check(self.kp.swap_in([i], [0, len(blocks)], np.array(blocks, np.int32)))
        kv.kv_check(self.kp.sync())
        self.table[i] = list(blocks)


def run(device="cuda", steps=90, preempt_at=30, seed=0):
    """-> (hidden states of the last step [n, width], tokens evicted, tokens read per cached token at the first step)"""
    s = Stream(torch.device(device, torch.cuda.current_device()), seed=seed)
    gen = torch.Generator(device="cpu").manual_seed(seed + 1)
    rand = lambda t: torch.randn(t, s.width, generator=gen).to(s.device, torch.bfloat16)  # noqa: E731
    prefix = 32 * s.g.B
    s.step([0], rand(prefix), [prefix])  # the system prompt, once
    for i in range(1, s.n):
        s.table[i], s.tokens[i], s.position[i] = list(s.table[0]), prefix, prefix
    prompts = [9 + 14 * i for i in range(s.n)]
    x = s.step(list(range(s.n)), rand(sum(prompts)), prompts)
    x = x[np.cumsum(prompts) - 1]
    share = None
    for t in range(steps):
        x = s.step(list(range(s.n)), torch.nn.functional.normalize(x.float(), dim=-1).bfloat16() * 16, [1] * s.n)
        info = s.batch.query()
        share = share or info["read_tokens"] / info["cached_tokens"]
        s.evict(prefix)
        if t == preempt_at:
            s.preempt(1)
            own = s.table[1][prefix // s.g.B:]
            s.pool.view(s.g.L, 2, s.g.N, -1)[:, :, torch.tensor([int(b) for b in own], device=s.device)] = 0xFF  # another owner's bytes
            torch.cuda.current_stream(s.device).synchronize()
            s.free = own + s.free
            s.resume(1, [s.free.pop() for _ in range(len(s.table[1]))])
    torch.cuda.synchronize()
    out, evicted = x.float().cpu(), s.evicted
    s.close()
    return out, evicted, share


def main():
    kept, evicted, share = run()
    plain, _, _ = run(preempt_at=-1)
    print("%d tokens evicted; a step reads %.0f %% of the cached tokens; preempted and resumed against undisturbed: %.2g apart (relative)" %
          (evicted, 100 * share, float((kept - plain).norm() / plain.norm())))


if __name__ == "__main__":
    main()
