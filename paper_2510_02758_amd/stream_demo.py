"""A small streaming decoder on the paged pool: the operators and the swap used together, as a serving loop would.

Several requests share a system prompt, whose blocks they have in common.  Each step sets the batch once; every layer turns and
appends the new tokens' keys, attends (the prefix read once for all) and accumulates what each cached token was given.  A
request that has grown past its budget gives up its lightest tokens in all layers, and the blocks behind the rest go back to the
free list.  One request is preempted on the way: swapped out, its blocks handed to others, and swapped into different ones later.

A second loop (speculate) drafts: after prompts with images, whose tokens have positions on three axes, each step sets a tree of guessed tokens for
every request, runs them all through the model at once, and keeps the path that the model agrees with.

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

    def forward(self, rows, x, new, where, pair_axes, parents=None):
        """The same with positions on several axes, where [axes, T], and without accumulated weights; parents: the new tokens are trees."""
        g, T = self.g, x.shape[0]
        off, ids = self._set(rows, new)
        if parents is not None:
            kv.kv_check(self.batch.set_trees(off, ids, [self.tokens[i] for i in rows], new, self.Hq, torch.tensor(parents, dtype=torch.int32, device=self.device)))
        where = torch.from_numpy(np.ascontiguousarray(where, np.int32)).to(self.device)
        out = torch.empty(T, self.Hq, g.D, dtype=torch.bfloat16, device=self.device)
        for layer in range(g.L):
            qkv = (x @ self.qkv[layer].t()).view(T, self.Hq + 2 * g.H, g.D)
            q, k, v = qkv[:, :self.Hq], qkv[:, self.Hq:self.Hq + g.H], qkv[:, self.Hq + g.H:]
            kv.kv_check(self.batch.append(layer, q, k, v, turns=self.turns, magnitude=self.magnitude, positions=where, pair_axes=pair_axes))
            kv.kv_check(self.batch.attn(layer, q, out, g.D ** -0.5))
            x = x + out.view(T, -1) @ self.proj[layer].t()
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


# A tree of eight drafts: parents, and which of its parent's likely successors a row is.  The last request's is smaller, padded to the same size.
PARENTS, GUESS = [-1, 0, 0, 0, 1, 1, 2, 4], [0, 0, 1, 2, 0, 1, 0, 0]
DEPTH = [0, 1, 1, 1, 2, 2, 2, 3]


def speculate(device="cuda", steps=20, seed=0):
    """-> per request: tokens [prompt and what followed], their positions [axes, tokens], hidden states of the tokens behind the prompt; accepted drafts a step"""
    s = Stream(torch.device(device, torch.cuda.current_device()), seed=seed)
    gen = torch.Generator(device="cpu").manual_seed(seed + 1)
    rand = lambda *z: torch.randn(*z, generator=gen).to(s.device, torch.bfloat16)  # noqa: E731
    words = 97
    embed, answer = rand(words, s.width), rand(words, s.width)
    likely = (embed.float() @ answer.float().t()).topk(3).indices.tolist()  # the drafter: what the model would say without its context
    pair_axes = np.array([0] * 8 + [1] * 12 + [2] * 12, np.int32)
    text, where, behind = [], [], []
    for i in range(s.n):  # some words, an image of 6 rows of patches, some words
        wide, t = 4 + i, 5 + i
        at = [[x] * 3 for x in range(t)] + [[t, t + r, t + c] for r in range(6) for c in range(wide)]
        behind.append(t + max(6, wide))
        at += [[behind[i] + x] * 3 for x in range(3)]
        behind[i] += 3
        where.append(at)
        text.append(torch.randint(0, words, (len(at),), generator=gen).tolist())
    rows, new = list(range(s.n)), [len(t) for t in text]
    x = s.forward(rows, embed[[t for r in text for t in r]], new, np.concatenate([np.array(w).T for w in where], 1), pair_axes)
    follows = (x[np.cumsum(new) - 1].float() @ answer.float().t()).argmax(-1).tolist()
    hidden, taken = [[] for _ in rows], []
    count, chosen_next = (torch.zeros(s.n, dtype=torch.int32, device=s.device) for _ in range(2))
    path = torch.zeros(s.n, len(PARENTS), dtype=torch.int32, device=s.device)
    for _ in range(steps):
        drafts, parents, at = [], [], []
        for i in rows:
            mine = [follows[i]]
            for p, k in zip(PARENTS[1:], GUESS[1:]):
                mine.append(likely[mine[p]][k])
            drafts += mine
            parents += PARENTS if i < s.n - 1 else PARENTS[:6] + [kv.KV_TREE_NONE] * 2
            at += [[behind[i] + d] * 3 for d in DEPTH]
        before = list(s.tokens)
        x = s.forward(rows, embed[drafts], [len(PARENTS)] * s.n, np.array(at).T, pair_axes, parents)
        chosen = (x.float() @ answer.float().t()).argmax(-1).to(torch.int32)
        kv.kv_check(s.batch.accept(0, s.g.L, torch.tensor(drafts, dtype=torch.int32, device=s.device), chosen, count, path, chosen_next, req_ids=rows))
        for i, (k, way) in enumerate(zip(count.tolist(), path.tolist())):  # (the host waits here for the step)
            for row in way[:k]:
                text[i].append(drafts[i * len(PARENTS) + row])
                where[i].append(at[i * len(PARENTS) + row])
                hidden[i].append(x[i * len(PARENTS) + row].float().cpu())
            s.tokens[i] = before[i] + k
            s.position[i] = behind[i] = behind[i] + k
            taken.append(k)
        follows = chosen_next.tolist()
    pool = s.pool.clone()
    # the same tokens one at a time, into a cache of their own
    plain = Stream(s.device, seed=seed)
    plain.forward(rows, embed[[t for r, n in zip(text, new) for t in r[:n]]], new, np.concatenate([np.array(w[:n]).T for w, n in zip(where, new)], 1), pair_axes)
    apart, size = 0.0, 0.0
    for j in range(min(len(h) for h in hidden)):
        x = plain.forward(rows, embed[[text[i][new[i] + j] for i in rows]], [1] * s.n, np.array([where[i][new[i] + j] for i in rows]).T, pair_axes).float().cpu()
        for i in rows:
            apart += float((hidden[i][j] - x[i]).square().sum())
            size += float(x[i].square().sum())
    # what is cached of them: rows of K and V, by the two tables
    g, rows_apart, rows_size = s.g, 0.0, 0.0
    steps_taken = min(len(h) for h in hidden)
    for i in rows:
        t = np.arange(new[i] + steps_taken)
        views = [m.view(torch.bfloat16).view(g.L, 2, g.N, g.B, g.H, g.D) for m in (pool, plain.pool)]
        a, b = (v[:, :, torch.from_numpy(np.asarray(tab, np.int64)[t // g.B]).to(s.device), torch.from_numpy(t % g.B).to(s.device)].float() for v, tab in
                zip(views, (s.table[i], plain.table[i])))
        rows_apart += float((a - b).square().sum())
        rows_size += float(b.square().sum())
    torch.cuda.synchronize()
    s.close()
    plain.close()
    return dict(accepted=sum(taken) / len(taken), hidden=(apart / size) ** 0.5, cache=(rows_apart / rows_size) ** 0.5, tokens=steps_taken)


def main():
    kept, evicted, share = run()
    plain, _, _ = run(preempt_at=-1)
    print("%d tokens evicted; a step reads %.0f %% of the cached tokens; preempted and resumed against undisturbed: %.2g apart (relative)" %
          (evicted, 100 * share, float((kept - plain).norm() / plain.norm())))
    drafted = speculate()
    print("drafts: %.2f tokens a request and step; against one token a step: hidden states %.2g, cached rows %.2g apart (relative)" %
          (drafted["accepted"], drafted["hidden"], drafted["cache"]))


if __name__ == "__main__":
    main()
