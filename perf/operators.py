"""What the operators on the paged KV pool are measured on: one call for one layer (eviction: for a range of layers) of a
serving loop, over the batches such a loop meets.

  append  rotary positions for queries and keys, with keys and values written into the blocks of the batch's requests
  attn    attention of the batch's new tokens over their requests' cached tokens, with prefixes that requests share; one
          query token a request (decode) or many (a prompt chunk); with or without accumulating what each cached token gets
  evict   the cached tokens with the largest accumulated weights stay, in order, at the front of their request's blocks

With `own` false the operators are computed in their plain form, in 32 bits, from elementary torch operations.  Shapes are
those of workloads.py and generic ones (odd head sizes and block sizes).
"""
import math

import torch

own = False

_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "fp8_e4m3": torch.float8_e4m3fn}


def _shape(L, H, D, B, dtype, G, scales=False):
    return dict(L=L, H=H, D=D, B=B, dtype=dtype, G=G, scales=scales)


_TINY = _shape(2, 4, 64, 16, "f16", 2)
_LLAMA8B = _shape(2, 8, 128, 16, "bf16", 4)
_LLAMA70B = _shape(2, 8, 128, 16, "bf16", 8)
_FP8_MHA = _shape(2, 32, 128, 32, "fp8_e4m3", 1, scales=True)
_ONE_HEAD = _shape(2, 1, 128, 16, "bf16", 8)


def _batch(n, lo, hi, q_lo=1, q_hi=1, prefix=0):
    """n requests of lo..hi tokens of their own behind `prefix` shared ones, the last q_lo..q_hi of them new."""
    return dict(n=n, lo=lo, hi=hi, q_lo=q_lo, q_hi=q_hi, prefix=prefix)


def _append(name, shape, batch, rot, interleaved, scaling):
    c = dict(op="append", **shape, **batch, rot=rot, interleaved=interleaved, scaling=scaling)
    return dict(c, name=name) if name else c


def _attn(name, shape, batch, weights=False):
    c = dict(op="attn", **shape, **batch, weights=weights)
    return dict(c, name=name) if name else c


def _evict(name, shape, batch, keep, first, last):
    c = dict(op="evict", **shape, **batch, keep=keep, first=first, last=last)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One decode step of a toy model: what a call costs.
        _append("tiny_append", _TINY, _batch(8, 16, 256), 64, True, "none"),
        # Three prompts of a model with stretched positions go into the cache.
        _append("llama8b_append_prompts", _LLAMA8B, _batch(3, 2000, 5001, 1031, 1801), 128, False, "parts"),
        # A decode step of a large batch on an fp8 pool with scales, half of each head rotated.
        _append("fp8_append_decode", _FP8_MHA, _batch(512, 64, 256), 64, False, "linear"),
        # One decode step of a toy model, one request still without a token: what a call costs.
        _attn("tiny_decode", _TINY, _batch(8, 0, 256)),
        # One decode step of a burst of ordinary requests.
        _attn("llama8b_decode_burst", _LLAMA8B, _batch(64, 512, 4096)),
        # One decode step of 128 requests behind one long system prompt.
        _attn("llama70b_shared_prefix", _LLAMA70B, _batch(128, 17, 900, prefix=8192)),
        # One decode step on an fp8 pool with scales, a query head for every KV head.
        _attn("fp8_decode", _FP8_MHA, _batch(32, 256, 8192)),
        # Two very long requests on a tensor-parallel shard with one KV head: few rows, a long axis.
        _attn("one_head_long_decode", _ONE_HEAD, _batch(2, 70001, 131072)),
        # Chunks of two prompts behind what is cached of them.
        _attn("llama8b_prompt_chunks", _LLAMA8B, _batch(2, 5000, 8001, 517, 1024)),
        # A decode step that also accumulates what every cached token was given.
        _attn("llama8b_decode_weights", _LLAMA8B, _batch(16, 300, 4096), weights=True),
        # Eviction on a toy model.
        _evict("tiny_evict", _TINY, _batch(8, 16, 256), 64, 4, 16),
        # Eight requests give up most of their tokens in all layers.
        _evict("llama8b_evict", dict(_LLAMA8B, L=32), _batch(8, 900, 2500), 512, 4, 128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    shape = rng.choice([_TINY, _LLAMA8B, _LLAMA70B, _FP8_MHA, _ONE_HEAD, None, None, None, None])
    if shape is None:
        dtype = rng.choice(["f16", "bf16", "fp8_e4m3"])
        shape = _shape(2, rng.choice([1, 2, 3, 4, 5, 8, 16]), rng.choice([64, 80, 96, 112, 128, 192, 256]), rng.choice([1, 4, 8, 16, 20, 32]), dtype,
                       rng.choice([1, 2, 3, 4, 5, 7, 8, 16]), scales=dtype == "fp8_e4m3" and rng.random() < 0.6)
    row = 2 * shape["H"] * shape["D"] * (1 if shape["dtype"] == "fp8_e4m3" else 2)  # bytes of a token in a layer
    op = rng.choice(["append", "append", "attn", "attn", "attn", "attn", "evict", "evict"])
    if op == "append":
        n = _log(rng, 1, 300)
        q = _log(rng, 1, max(1, min(4000, 4500 // n))) if rng.random() < 0.5 else 1
        rot = shape["D"] if rng.random() < 0.6 else 2 * rng.randint(1, shape["D"] // 2)
        hi = q + _log(rng, 1, 500)
        return _append(None, shape, _batch(n, rng.randint(q, hi), hi, rng.randint(1, q), q), rot, rng.random() < 0.5, rng.choice(["none", "linear", "parts", "yarn"]))
    if op == "evict":
        tokens = _log(rng, 64, max(65, min(1 << 17, (1 << 28) // row)))
        n = min(_log(rng, 1, 16), tokens // 32)
        hi = tokens // n
        shape = dict(shape, L=2 * rng.randint(1, max(1, min(16, (1 << 28) // (row * tokens)))))
        first, last = rng.choice([0, 4, 17]), rng.choice([0, 1, 32])
        return _evict(None, shape, _batch(n, rng.randint(1, hi), hi), first + last + _log(rng, 1, max(2, 3 * hi // 4)), first, last)
    rows = shape["H"] * shape["G"]
    if rng.random() < 0.3:  # a prompt chunk
        n, q = rng.choice([1, 1, 2, 3]), _log(rng, 2, 700)
        hi = q + _log(rng, 1, max(2, min(8000, int(6e10 / (4.0 * n * q * rows * shape["D"])))))
        return _attn(None, shape, _batch(n, rng.randint(q, hi), hi, rng.randint(1, q), q), rng.random() < 0.2)
    if rng.random() < 0.35:  # many requests behind one prefix
        n = _log(rng, 2, 100)
        own_hi = _log(rng, 2, max(3, min(1000, (1 << 28) // (row * n))))
        prefix = _log(rng, 32, max(33, min(8192, int(8e9 / (8.0 * n * shape["H"] * shape["D"]) - own_hi))))
        return _attn(None, shape, _batch(n, rng.randint(1, own_hi), own_hi, prefix=max(1, prefix // shape["B"]) * shape["B"]), rng.random() < 0.2)
    n = _log(rng, 1, 200)
    hi = _log(rng, 8, max(9, min(100000, (1 << 29) // (row * n))))
    q = rng.choice([1, 1, 1, 2, 4])
    q = min(q, hi)
    return _attn(None, shape, _batch(n, rng.randint(0 if q == 1 else q, hi), hi, rng.randint(1, q), q), rng.random() < 0.3)


# ------------------------------------------------------------------ sizes of a case (the same for every seed)

def _between(n, lo, hi, step):
    """n whole numbers spread evenly over lo..hi, both reached, in a mixed order."""
    if n == 1:
        return [hi]
    while math.gcd(step, n) > 1:
        step += 1
    return [lo + (hi - lo) * ((i * step) % n) // (n - 1) for i in range(n)]


def _lengths(case):
    """Per request: cached tokens with the shared ones and the new ones, new ones (at least one, and at most what the request has
    of its own; a request without any token still has one row)."""
    lens = _between(case["n"], case["lo"], case["hi"], 7)
    new = _between(case["n"], case["q_lo"], case["q_hi"], 5)
    new = [max(1, min(q, x)) for q, x in zip(new, lens)]
    return [case["prefix"] + x for x in lens], new


def _elem(case):
    return 1 if case["dtype"] == "fp8_e4m3" else 2


def work(case):
    lens, new = _lengths(case)
    H, D, G, e = case["H"], case["D"], case["G"], _elem(case)
    T = sum(new)
    if case["op"] == "append":  # q in and out, k and v in and out
        return {"bytes": T * D * (2 * H * G * 2 + 2 * H * (2 + e)), "flops": 3 * T * (H * G + H) * case["rot"]}
    if case["op"] == "attn":
        tokens = case["prefix"] + sum(x - case["prefix"] for x in lens)
        pairs = sum(q * max(0, x - q) + q * (q + 1) // 2 if x >= q else 0 for x, q in zip(lens, new))
        nbytes = tokens * 2 * H * D * e + T * H * G * (2 * 2 * D + 4)
        if case["scales"]:
            nbytes += -(-tokens // case["B"]) * 2 * H * 4
        if case["weights"]:
            nbytes += sum(lens) * H * 8
        return {"bytes": nbytes, "flops": 4 * pairs * H * G * D}
    heads, nbytes = case["L"] * H, 0
    for x in lens:
        k = min(x, case["keep"])
        nbytes += heads * (8 * x + 4 * k)
        if x > k:
            nbytes += heads * (k - min(k, case["first"])) * 2 * 2 * D * e
    return {"bytes": nbytes, "flops": 0}


# ------------------------------------------------------------------ rotary frequencies

def _frequencies(rot, scaling):
    """(turns a position for each of the rot / 2 pairs, magnitude of cosines and sines): the usual scalings for long contexts."""
    base, factor, trained = 500000.0, 8.0, 8192.0
    f = [base ** (-2.0 * j / rot) / (2 * math.pi) for j in range(rot // 2)]
    if scaling == "linear":
        return [x / factor for x in f], 1.0
    if scaling == "parts":  # pairs that turn often stay, slow ones are stretched, between them a ramp over turns within the trained length
        out = []
        for x in f:
            mix = min(1.0, max(0.0, (trained * x - 1.0) / (4.0 - 1.0)))
            out.append((1 - mix) * x / factor + mix * x)
        return out, 1.0
    if scaling == "yarn":  # a ramp over the pairs' indices, and larger logits
        def at(turns):
            return rot * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base))
        low, high = max(0.0, math.floor(at(32.0))), min(rot - 1.0, math.ceil(at(1.0)))
        high = high + 0.001 if high == low else high
        out = []
        for j, x in enumerate(f):
            ramp = min(1.0, max(0.0, (j - low) / (high - low)))
            out.append(x / factor * ramp + x * (1 - ramp))
        return out, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _fixed(f):
    """Turns in units of 2^-64, as signed 64-bit words: products with a position wrap around once a turn."""
    out = []
    for x in f:
        w = int(round(math.ldexp(math.fmod(x, 1.0), 64))) & ((1 << 64) - 1)
        out.append(w - (1 << 64) if w >> 63 else w)
    return out


# ------------------------------------------------------------------ inputs

class _State:
    pass


def _fill(x, gen, dtype, size):
    """Normal values of standard deviation `size`."""
    if dtype == "fp8_e4m3":
        x.copy_((torch.randn(x.shape, generator=gen, device="cuda", dtype=torch.bfloat16) * size).clamp_(-448, 448))
    else:
        x.normal_(0.0, size, generator=gen)


def prepare(case, seed):
    s = _State()
    s.case = c = case
    L, H, D, B, G = (c[k] for k in ("L", "H", "D", "B", "G"))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    host = torch.Generator()
    host.manual_seed(int(seed))
    s.lens, s.new = _lengths(c)
    T = sum(s.new)
    shared = c["prefix"] // B
    rows = [-(-(x - c["prefix"]) // B) for x in s.lens]
    used = shared + sum(rows)
    N = used + 1 + used // 8
    perm = torch.randperm(N, generator=host, dtype=torch.int64).to(torch.int32)
    ids, off, at = [], [0], shared
    for r in rows:
        ids.append(torch.cat([perm[:shared], perm[at:at + r]]))
        at += r
        off.append(off[-1] + shared + r)
    s.ids, s.off = torch.cat(ids).numpy(), torch.tensor(off, dtype=torch.int32).numpy()
    dtype = _DTYPE[c["dtype"]]
    s.io = torch.bfloat16 if c["dtype"] != "f16" else torch.float16
    s.pool = torch.empty(L, 2, N, B, H, D, dtype=dtype, device="cuda")
    for layer in range(L):
        _fill(s.pool[layer], gen, c["dtype"], 40.0 if c["dtype"] == "fp8_e4m3" else 1.0)
    s.scale = torch.empty(L, 2, N, H, device="cuda").uniform_(0.02, 0.03, generator=gen) if c["scales"] else None
    s.layer = L - 1

    # what the plain form and the library's handle need of the batch, on the GPU: the table row by row, padded
    width = max(off[i + 1] - off[i] for i in range(c["n"])) if c["n"] else 0
    table = torch.zeros(c["n"], max(1, width), dtype=torch.int64)
    for i in range(c["n"]):
        table[i, :off[i + 1] - off[i]] = torch.from_numpy(s.ids[off[i]:off[i + 1]]).long()
    s.table = table.cuda()
    s.len = torch.tensor(s.lens, device="cuda")
    s.q_len = torch.tensor(s.new, device="cuda")
    s.max_len, s.max_q = max(s.lens), max(s.new)
    first = torch.tensor([0] + s.new[:-1]).cumsum(0)
    s.first_row = first.cuda()
    req = torch.repeat_interleave(torch.arange(c["n"]), torch.tensor(s.new))
    s.req = req.cuda()
    s.index = (torch.tensor(s.lens)[req] - torch.tensor(s.new)[req] + torch.arange(T) - first[req]).cuda()  # place in the cache; -1: none

    if c["op"] == "append":
        # new tokens come out of one projection: queries, keys and values side by side
        s.qkv = torch.empty(T, (G + 2) * H, D, dtype=s.io, device="cuda").normal_(0.0, 1.0, generator=gen)
        s.q, s.k, s.v = s.qkv[:, :G * H], s.qkv[:, G * H:(G + 1) * H], s.qkv[:, (G + 1) * H:]
        s.q_out = torch.empty(T, G * H, D, dtype=s.io, device="cuda")
        f, s.magnitude = _frequencies(c["rot"], c["scaling"])
        s.turns = torch.tensor(_fixed(f), dtype=torch.int64, device="cuda")
        # a cache from which tokens were evicted: positions run ahead of the places
        ahead = torch.randint(0, 20000, (c["n"],), generator=host)
        s.positions = (s.index + ahead.cuda()[s.req]).to(torch.int32)
        s.kv_scale = torch.empty(2, H, device="cuda").uniform_(0.01, 0.02, generator=gen) if c["scales"] else None
    elif c["op"] == "attn":
        s.q = torch.empty(T, G * H, D, dtype=s.io, device="cuda").normal_(0.0, 2.0, generator=gen)
        s.out = torch.empty(T, G * H, D, dtype=s.io, device="cuda")
        s.lse = torch.empty(T, G * H, device="cuda")
        s.softmax_scale = D ** -0.5
        s.weights = torch.empty(c["n"], H, s.max_len, device="cuda").uniform_(0.0, 1.0, generator=gen) if c["weights"] else None
    else:
        # accumulated weights fall off steeply; tokens that nothing has looked at yet have exactly 0
        w = torch.empty(L, c["n"], H, s.max_len, device="cuda").uniform_(0.0, 1.0, generator=gen)
        s.weights = torch.where(w < 0.1, torch.zeros_like(w), w.pow(8.0))
        s.weights_out = torch.zeros_like(s.weights)  # the accumulators that the following steps go on with: a pass can be repeated
        s.kept = torch.full((L, c["n"], H, c["keep"]), -1, dtype=torch.int32, device="cuda")
        s.crowded = torch.tensor([i for i, x in enumerate(s.lens) if x > c["keep"]], dtype=torch.int64, device="cuda")
    if own:
        _handle(s, N)
    return s


def _handle(s, N):
    """The handle on the pool and the batch that a serving loop keeps: the batch is set once a step and used by every layer."""
    from paper_2510_02758_amd import kvswap as kv
    from paper_2510_02758_amd import workloads as W
    c = s.case
    g = W.Geometry(c["L"], c["H"], c["D"], c["B"], c["dtype"], N, scales=c["scales"])
    arena = torch.empty(g.S, dtype=torch.uint8, device="cuda")
    s.kp = kv.KVPool(g, s.pool.view(torch.uint8).reshape(-1), arena, scale=None if s.scale is None else s.scale.view(torch.uint8).reshape(-1),
                     flags=kv.KV_STAGING_DEVICE)
    s.batch = kv.KVBatch(s.kp)
    s.ok = kv.kv_check
    s.ok(s.batch.set(s.off, s.ids, s.lens, s.new, c["G"] * c["H"]))


# ------------------------------------------------------------------ one pass

def run(s):
    c = s.case
    if c["op"] == "append":
        if own:
            ks, vs = (None, None) if s.kv_scale is None else (s.kv_scale[0], s.kv_scale[1])
            s.ok(s.batch.append(s.layer, s.q, s.k, s.v, s.q_out, turns=s.turns, interleaved=c["interleaved"], magnitude=s.magnitude,
                                positions=s.positions, k_scale=ks, v_scale=vs))
        else:
            _append_plain(s)
        out = {"q": s.q_out, "pool": s.pool}
        if s.scale is not None:
            out["scale"] = s.scale
        return out
    if c["op"] == "attn":
        if own:
            s.ok(s.batch.attn(s.layer, s.q, s.out, s.softmax_scale, lse=s.lse, weights=s.weights))
        else:
            _attn_plain(s)
        out = {"out": s.out, "lse": s.lse}
        if s.weights is not None:
            out["weights"] = s.weights
        return out
    if own:
        s.ok(s.batch.evict(0, c["L"], s.weights, s.kept, c["keep"], keep_first=c["first"], keep_last=c["last"],
                         weights_out=s.weights_out))
    else:
        _evict_plain(s)
    out = {"kept": s.kept, "weights": s.weights_out, "pool": s.pool}
    if s.scale is not None:
        out["scale"] = s.scale
    return out


def _rotate(x, cos, sin, rot, interleaved):
    x = x.float()
    a, b = (x[..., :rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    cos, sin = cos[:, None], sin[:, None]
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _append_plain(s):
    c = s.case
    phase = s.positions.long()[:, None] * s.turns[None]  # wraps once a turn
    angle = (phase >> 40).float() * (2 * math.pi / (1 << 24))
    cos, sin = angle.cos() * s.magnitude, angle.sin() * s.magnitude
    s.q_out.copy_(_rotate(s.q, cos, sin, c["rot"], c["interleaved"]))
    k, v = _rotate(s.k, cos, sin, c["rot"], c["interleaved"]), s.v.float()
    block, place = s.table[s.req, s.index // c["B"]], s.index % c["B"]
    if s.kv_scale is not None:
        k, v = k / s.kv_scale[0][:, None], v / s.kv_scale[1][:, None]
        s.scale[s.layer, 0, block] = s.kv_scale[0]
        s.scale[s.layer, 1, block] = s.kv_scale[1]
    if c["dtype"] == "fp8_e4m3":  # assigned as the bytes that they are
        k, v = (x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for x in (k, v))
    pool = s.pool.view(torch.uint8) if c["dtype"] == "fp8_e4m3" else s.pool
    pool[s.layer, 0, block, place] = k.to(pool.dtype)
    pool[s.layer, 1, block, place] = v.to(pool.dtype)


def _gathered(s, which):
    """The batch's keys or values of the layer as (request, head, place, D) in 32 bits, zero behind each request's last."""
    c = s.case
    x = torch.arange(s.max_len, device="cuda")
    block = s.table[:, x // c["B"]]
    pool = s.pool[s.layer, which]
    pool = pool.view(torch.uint8) if c["dtype"] == "fp8_e4m3" else pool  # gathered as the bytes that they are
    rows = pool[block, x % c["B"]].view(s.pool.dtype).float()
    if s.scale is not None:
        rows = rows * s.scale[s.layer, which][block][..., None]
    return torch.where((x[None] < s.len[:, None])[..., None, None], rows, torch.zeros_like(rows)).transpose(1, 2)


def _attn_plain(s):
    c = s.case
    n, H, G, D = c["n"], c["H"], c["G"], c["D"]
    j = torch.arange(s.max_q, device="cuda")
    real = j[None] < s.q_len[:, None]
    row = torch.where(real, s.first_row[:, None] + j[None], torch.zeros_like(s.first_row)[:, None])
    q = s.q[row].float().view(n, s.max_q, H, G, D).permute(0, 2, 1, 3, 4).reshape(n, H, s.max_q * G, D)
    x = torch.arange(s.max_len, device="cuda")
    last = (s.len - s.q_len)[:, None] + j[None]
    seen = ((x[None, None] <= last[..., None]) & real[..., None])[:, None, :, None]  # (n, 1, max_q, 1, max_len)
    z = torch.matmul(q, _gathered(s, 0).transpose(2, 3)).view(n, H, s.max_q, G, s.max_len) * s.softmax_scale
    z = z.masked_fill(~seen, -math.inf)
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(m == -math.inf, torch.zeros_like(m), m))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    o = torch.matmul(p.view(n, H, s.max_q * G, s.max_len), _gathered(s, 1)).view(n, H, s.max_q, G, D)
    lse = (m + torch.log(total))[..., 0]
    i, t = s.req, s.index - (s.len - s.q_len)[s.req]
    s.out.copy_(o[i, :, t].reshape(-1, H * G, D))
    s.lse.copy_(lse[i, :, t].reshape(-1, H * G))
    if s.weights is not None:
        s.weights += p.sum((2, 3))


def _evict_plain(s):
    c = s.case
    L, n, H, D, B = c["L"], c["n"], c["H"], c["D"], c["B"]
    x = torch.arange(s.max_len, device="cuda")
    free = (x[None] >= c["first"]) & (x[None] < s.len[:, None] - c["last"])  # tokens that may go
    rank = torch.where(free, s.weights.transpose(1, 2), torch.full((), math.inf, device="cuda"))
    rank = torch.where(x[None] < s.len[:, None], rank, torch.full((), -math.inf, device="cuda"))  # (L, H, n, max_len)
    order = rank.sort(dim=-1, descending=True, stable=True).indices[..., :min(c["keep"], s.max_len)]
    kept = order.sort(-1).values.transpose(1, 2)  # (L, n, H, k): places in order
    k = kept.shape[-1]
    crowded = (s.len > c["keep"])[None, :, None, None]
    place = torch.arange(k, device="cuda")
    kept = torch.where(crowded, kept, place)
    inside = place[None] < s.len[:, None]
    s.kept[..., :k] = torch.where(inside[None, :, None], kept, s.kept[..., :k].long()).to(torch.int32)
    w = torch.zeros_like(s.weights)
    w[..., :k] = s.weights.gather(-1, kept)
    s.weights_out.copy_(torch.where((x[None] < s.len[:, None])[None, :, None], torch.where(crowded, w, s.weights), s.weights_out))
    # rows that move, as bytes: those of the crowded requests
    which = s.crowded
    if not len(which):
        return
    kept = kept[:, which]
    table = s.table[which]
    layer, head = torch.arange(L, device="cuda").view(L, 1, 1, 1), torch.arange(H, device="cuda").view(1, 1, H, 1)
    src = table.view(1, len(which), 1, -1).expand(L, -1, H, -1).gather(-1, kept // B)
    dst = table[:, place // B].view(1, len(which), 1, k).expand(L, -1, H, -1)
    pool = s.pool.view(torch.uint8) if c["dtype"] == "fp8_e4m3" else s.pool
    if s.scale is None:
        for kv in range(2):
            pool[layer, kv, dst, place % B, head] = pool[layer, kv, src, kept % B, head]
        return
    # with scales, a block's new one is the largest that its tokens come with, and tokens that come with less are rounded again
    for kv in range(2):
        rows = pool[layer, kv, src, kept % B, head]
        old = s.scale[layer, kv, src, head]
        new = torch.zeros(L, len(which), H, -(-k // B), device="cuda").scatter_reduce(-1, (place // B).expand(L, len(which), H, k), old, "amax")
        new_row = new[..., place // B]
        again = (rows.view(torch.float8_e4m3fn).float() * (old / new_row)[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        pool[layer, kv, dst, place % B, head] = torch.where((old == new_row)[..., None], rows, again)
        s.scale[layer, kv, dst, head] = new_row


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    if case["op"] == "evict":
        return None  # tokens are moved, nothing is computed
    s = prepare(case, seed)
    return _append_exact(s) if case["op"] == "append" else _attn_exact(s)


def _append_exact(s):
    c = s.case
    rot, B = c["rot"], c["B"]
    f, magnitude = _frequencies(rot, c["scaling"])
    turns = s.positions.double()[:, None] * torch.tensor(f, dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.full_like(turns, magnitude), 2 * math.pi * (turns - turns.round()))[:, None]

    def rotated(x):
        x = x.double()
        y = x.clone()
        if c["interleaved"]:
            z = torch.complex(x[..., 0:rot:2], x[..., 1:rot:2]) * turn
            y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
        else:
            z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
            y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
        return y

    pool = s.pool.double()
    scale = None if s.scale is None else s.scale.double()
    block, place = s.table[s.req, s.index // B], s.index % B
    for kv, x in ((0, rotated(s.k)), (1, s.v.double())):
        if scale is not None:
            x = x / s.kv_scale[kv].double()[:, None]
            scale[s.layer, kv, block] = s.kv_scale[kv].double()
        pool[s.layer, kv, block, place] = x.clamp(-448, 448) if c["dtype"] == "fp8_e4m3" else x
    out = {"q": rotated(s.q), "pool": pool}
    if scale is not None:
        out["scale"] = scale
    return out


def _attn_exact(s):
    c = s.case
    H, G, D, B = c["H"], c["G"], c["D"], c["B"]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s.lse.shape, -math.inf, dtype=torch.float64, device="cuda")
    weights = None if s.weights is None else s.weights.double()
    t = 0
    for i, (length, new) in enumerate(zip(s.lens, s.new)):
        rows = s.q[t:t + new].double().view(new, H, G, D)
        blocks = s.table[i, :-(-length // B)]
        if length:
            for h in range(H):
                kv = s.pool[s.layer][:, blocks, :, h].double() if c["dtype"] != "fp8_e4m3" else \
                    s.pool.view(torch.uint8)[s.layer][:, blocks, :, h].contiguous().view(torch.float8_e4m3fn).double()
                if s.scale is not None:
                    kv = kv * s.scale[s.layer][:, blocks, h].double()[..., None, None]
                kv = kv.reshape(2, -1, D)[:, :length]
                z = torch.tensordot(rows[:, h], kv[0].t().contiguous(), 1) * s.softmax_scale
                hidden = torch.ones(new, length, dtype=torch.bool, device="cuda").triu(length - new + 1)
                z.masked_fill_(hidden[:, None], -math.inf)
                l = z.logsumexp(-1)
                p = (z - l[..., None]).exp()
                out[t:t + new].view(new, H, G, D)[:, h] = torch.tensordot(p, kv[1].contiguous(), 1)
                lse[t:t + new].view(new, H, G)[:, h] = l
                if weights is not None:
                    weights[i, h, :length] += p.sum((0, 1))
        t += new
    res = {"out": out, "lse": lse}
    if weights is not None:
        res["weights"] = weights
    return res
