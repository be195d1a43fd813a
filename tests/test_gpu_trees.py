"""Drafted trees over the paged pool (attention, positions, the accepted path) and rotary positions with several axes on a real MI355X, against plain
implementations in 64 bits (trees_ref.py)."""
import numpy as np
import pytest

import ops_ref as R
import trees_ref as TR
from paper_2510_02758_amd import kvswap as kv
from paper_2510_02758_amd import workloads as W
from test_gpu_ops import Pool, _heads, _tables, _torch_type

pytestmark = pytest.mark.gpu


def _parents(rng, q, kind):
    """Parents of a tree of q rows."""
    if kind == "chain":
        return [TR.ROOT] + list(range(q - 1))
    if kind == "star":
        return [TR.ROOT] + [0] * (q - 1)
    if kind == "roots":                       # nothing in front but the cache
        return [TR.ROOT] * q
    if kind == "none":                        # no row is in the tree
        return [TR.NONE] * q
    if kind == "last alone":                  # only the last row is
        return [TR.NONE] * (q - 1) + [TR.ROOT]
    if kind == "strange":                     # numbers that are no parent: itself, behind it, below KV_TREE_NONE, and descendants of these
        out = [TR.ROOT]
        for j in range(1, q):
            out.append(int(rng.choice([j, j + 1, q, -7, -2 ** 31, 2 ** 31 - 1]) if rng.random() < 0.2 else rng.integers(-1, j)))
        return out
    out = [TR.ROOT]
    for j in range(1, q):
        out.append(int(rng.integers(max(0, j - 6), j)))
    if kind == "padded":
        out[q - q // 3:] = [TR.NONE] * (q // 3)
    return out


# name: geometry (L, H, D, B, dtype, scales), G, lens, q_lens, kinds ("-": the new tokens follow one another), shared, layout, (pad, off)
TREES = {
    "one row": ((1, 1, 64, 16, "bf16", False), 1, [1], [1], ["chain"], (), "layer", (0, 0)),
    "nothing cached": ((2, 2, 64, 16, "f16", False), 2, [0, 0, 5], [1, 0, 5], ["chain", "chain", "random"], (), "layer", (0, 0)),
    "nothing in front": ((1, 2, 64, 16, "bf16", False), 2, [9, 40, 1], [9, 40, 1], ["random", "padded", "none"], (), "layer", (0, 0)),
    "few rows": ((2, 4, 64, 16, "f16", False), 2, [15, 16, 17, 31, 33, 64, 65, 127, 128, 129, 300], [2, 3, 4, 5, 6, 7, 8, 1, 2, 3, 4],
                 ["random", "star", "chain", "padded", "roots", "strange", "random", "none", "last alone", "padded", "random"], (), "layer", (0, 0)),
    "trees and others": ((1, 2, 128, 16, "bf16", False), 4, [600, 300, 77, 500, 41, 40], [8, 130, 1, 33, 1, 3], ["random", "-", "-", "padded", "chain", "-"], (),
                         "layer", (0, 0)),
    "requests without a row": ((1, 2, 128, 16, "bf16", False), 4, [40, 100, 7, 60], [0, 1, 0, 9], ["random", "chain", "-", "random"], (), "layer", (0, 0)),
    "32 rows": ((1, 2, 128, 16, "bf16", False), 4, [700, 90, 333], [8, 8, 8], ["random", "padded", "strange"], (), "layer", (0, 0)),
    "a tile and more": ((1, 2, 128, 16, "f16", False), 4, [900, 200], [40, 33], ["random", "strange"], (), "block", (0, 0)),
    "17 rows": ((1, 2, 128, 32, "bf16", False), 1, [900, 200], [17, 17], ["random", "strange"], (), "layer", (0, 0)),
    "odd heads": ((2, 3, 72, 5, "bf16", False), 5, [9, 77, 200], [3, 20, 7], ["random", "padded", "random"], (), "layer", (8, 8)),
    "d 80, strides of 2 bytes": ((1, 2, 80, 16, "f16", False), 3, [90, 333], [5, 40], ["random", "padded"], (), "block", (3, 5)),
    "d 96, blocks of one": ((1, 2, 96, 1, "bf16", False), 7, [300, 40], [2, 30], ["star", "strange"], (), "layer", (0, 0)),
    "d 192": ((1, 2, 192, 16, "bf16", False), 2, [400, 60], [7, 50], ["random", "padded"], (), "layer", (0, 0)),
    "d 256, blocks of 20": ((1, 1, 256, 20, "f16", False), 8, [500, 41], [2, 12], ["roots", "random"], (), "layer", (0, 0)),
    "d 256, blocks of 16": ((2, 2, 256, 16, "bf16", False), 4, [300, 77], [4, 70], ["random", "strange"], (), "layer", (0, 0)),
    "d 8": ((1, 2, 8, 8, "bf16", False), 2, [70], [9], ["random"], (), "layer", (0, 0)),
    "many query heads": ((1, 1, 128, 16, "bf16", False), 71, [290, 45], [3, 2], ["star", "padded"], (), "layer", (0, 0)),
    "more query heads than a tile has rows": ((1, 1, 64, 16, "bf16", False), 150, [290, 45, 30], [3, 2, 4], ["star", "padded", "-"], (), "layer", (0, 0)),
    "long, few rows": ((1, 1, 128, 16, "bf16", False), 2, [20011], [8], ["random"], (), "layer", (0, 0)),
    "long, many rows": ((1, 1, 128, 16, "bf16", False), 8, [20011], [48], ["random"], (), "layer", (0, 0)),
    "long, token by token": ((1, 1, 64, 1, "f16", False), 4, [9001], [13], ["random"], (), "layer", (0, 0)),
    "the largest tree": ((1, 1, 64, 16, "bf16", False), 1, [1500, 1024], [1024, 1024], ["random", "chain"], (), "layer", (0, 0)),
    "a large tree in odd blocks": ((1, 1, 64, 7, "f16", False), 2, [1100], [515], ["strange"], (), "layer", (0, 0)),
    "fp8": ((2, 2, 128, 32, "fp8_e4m3", False), 4, [50, 700], [3, 9], ["random", "padded"], (), "layer", (0, 0)),
    "fp8 with scales": ((2, 4, 128, 32, "fp8_e4m3", True), 1, [257, 64, 1000, 90], [17, 8, 31, 64], ["random", "padded", "strange", "random"], (), "layer", (0, 0)),
    "fp8 with scales, odd": ((2, 2, 72, 6, "fp8_e4m3", True), 3, [257, 64, 5], [30, 3, 2], ["random", "star", "padded"], (), "layer", (1, 1)),
    "fp8 with scales, d 64": ((2, 2, 64, 16, "fp8_e4m3", True), 9, [100, 511], [2, 1], ["star", "chain"], (), "block", (0, 0)),
    "fp8 d 256": ((2, 1, 256, 16, "fp8_e4m3", True), 4, [100, 511], [40, 2], ["random", "star"], (), "layer", (0, 0)),
    "behind a prefix": ((1, 2, 128, 16, "bf16", False), 4, [1100, 1200, 1060, 1055], [9, 16, 1, 4], ["random", "padded", "none", "strange"],
                        ((1, 0, 65), (2, 0, 65), (3, 0, 65)), "layer", (0, 0)),
    "many behind a prefix": ((1, 8, 128, 16, "bf16", False), 4, [2100 + 7 * i for i in range(33)], [1 + i % 9 for i in range(33)],
                             [["random", "padded", "-", "none", "strange"][i % 5] for i in range(33)], tuple((i, 0, 128) for i in range(1, 33)), "layer", (0, 0)),
    "fp8 behind a prefix": ((1, 8, 64, 16, "fp8_e4m3", True), 4, [2100 + 7 * i for i in range(40)], [1 + i % 6 for i in range(40)],
                            [["random", "padded", "star"][i % 3] for i in range(40)], tuple((i, 0, 128) for i in range(1, 40)), "layer", (0, 0)),
}


def _drafts(gpu, name, seed=0):
    """-> pool, tables, parents of each request (None: no tree), the device's parents, queries"""
    import torch
    (L, H, D, B, dtype, scales), G, lens, q_lens, kinds, shared, layout, (pad, off) = TREES[name]
    N = sum(-(-n // B) for n in lens) + 3
    p = Pool(gpu, W.Geometry(L, H, D, B, dtype, N, scales=scales), layout, seed=len(name) + seed)
    rows = _tables(p.rng, N, lens, B, shared)
    p.fill(rows, lens)
    trees = [None if k == "-" else _parents(p.rng, q, k)[:q] for k, q in zip(kinds, q_lens)]
    every = [x for t, q in zip(trees, q_lens) for x in (t if t is not None else [12345] * q)]  # (what belongs to no tree is not looked at)
    parents = torch.tensor(every, dtype=torch.int64).to(torch.int32).to(gpu)
    return p, rows, trees, parents


def _spoil_rows_of_no_tree(p, rows, lens, q_lens, trees, q):
    """What nobody may look at holds NaN: keys, values and queries of rows that are in no tree."""
    nan = {"fp8_e4m3": 0x7F, "bf16": 0x7FC1, "f16": 0x7E01}[p.g.dtype]
    t = 0
    for table, n, new, tree in zip(rows, lens, q_lens, trees):
        if tree is not None and n:
            inside, _ = TR.ancestry(tree)
            for j in np.nonzero(~inside)[0]:
                x = n - new + j
                p.bits()[:, :, int(table[x // p.g.B]), x % p.g.B] = nan
                q[t + int(j)] = float("nan")
        t += new


@pytest.mark.parametrize("name", list(TREES))
def test_tree_attention(gpu, name):
    import torch
    (L, H, D, B, dtype, _), G, lens, q_lens, kinds, _, _, (pad, off) = TREES[name]
    p, rows, trees, parents = _drafts(gpu, name)
    T, layer, scale = sum(q_lens), L - 1, 1.3 * D ** -0.5
    o, ids = R.csr(rows)
    for io_name in ([dtype] if dtype != "fp8_e4m3" else ["bf16", "f16"]):
        io = _torch_type(io_name)
        q = _heads(torch, gpu, p.rng.standard_normal((T, G * H, D)) * (1.0 if dtype != "fp8_e4m3" else 0.1), io, pad, off)
        ref, tol, rlse, ltol, rw, wtol = TR.attention(p.values()[layer], rows, lens, q_lens, trees, q.double().cpu().numpy(), scale, io_name, B)
        _spoil_rows_of_no_tree(p, rows, lens, q_lens, trees, q)
        out = _heads(torch, gpu, np.zeros((T, G * H, D)), io, pad, off)
        lse = torch.full((T, G * H + 1), 7.0, device=gpu)[:, :G * H]
        start = torch.rand(len(lens), H, max(lens) + 3, device=gpu)
        weights = start.clone()
        kv.kv_check(p.batch.set_trees(o, ids, lens, q_lens, G * H, parents, [t is not None for t in trees]))
        kv.kv_check(p.batch.attn(layer, q, out, scale, lse=lse, weights=weights))
        again, lse2 = torch.empty_like(out), torch.empty(T, G * H, device=gpu)
        kv.kv_check(p.batch.attn(layer, q, again, scale, lse=lse2))
        torch.cuda.synchronize()
        got = out.double().cpu().numpy()
        assert (np.abs(got - ref) <= tol).all(), np.nanmax(np.abs(got - ref) - tol)
        gl = lse.double().cpu().numpy()
        dead = rlse == -np.inf
        assert (gl[dead] == -np.inf).all() and (np.abs(gl[~dead] - rlse[~dead]) <= ltol[~dead]).all()
        assert torch.equal(again, out) and torch.equal(lse2, lse)
        for i, n in enumerate(lens):
            added = (weights[i, :, :n].double() - start[i, :, :n].double()).cpu().numpy()
            slack = (2.0 ** -22 * (1 + np.abs(rw[i])) + wtol[i]) * (1 + q_lens[i])
            assert (np.abs(added - rw[i]) <= slack).all(), i
            assert torch.equal(weights[i, :, n:], start[i, :, n:])


@pytest.mark.parametrize("name", ["few rows", "32 rows", "fp8 with scales", "behind a prefix"])
def test_captured_weights(gpu, name):
    """The first call that wants weights is in a capture: there is no room for products, which are computed again."""
    import torch
    (L, H, D, B, dtype, _), G, lens, q_lens, *_ = TREES[name]
    p, rows, trees, parents = _drafts(gpu, name)
    o, ids = R.csr(rows)
    io_name = "f16" if dtype == "f16" else "bf16"
    q = torch.from_numpy(p.rng.standard_normal((sum(q_lens), G * H, D)) * (1.0 if dtype != "fp8_e4m3" else 0.1)).to(_torch_type(io_name)).to(gpu)
    ref, tol, _, _, rw, wtol = TR.attention(p.values()[L - 1], rows, lens, q_lens, trees, q.double().cpu().numpy(), D ** -0.5, io_name, B)
    _spoil_rows_of_no_tree(p, rows, lens, q_lens, trees, q)
    out, weights = torch.empty_like(q), torch.zeros(len(lens), H, max(lens), device=gpu)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    kv.kv_check(p.batch.set_trees(o, ids, lens, q_lens, G * H, parents, [t is not None for t in trees], stream=st))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        kv.kv_check(p.batch.attn(L - 1, q, out, D ** -0.5, weights=weights, stream=st))
    for turn in range(3):
        weights.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            graph.replay()
        st.synchronize()
        assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()
        for i, n in enumerate(lens):
            assert (np.abs(weights[i, :, :n].double().cpu().numpy() - rw[i]) <= (2.0 ** -22 * (1 + np.abs(rw[i])) + wtol[i]) * (1 + q_lens[i])).all(), (turn, i)


def test_far_into_a_pool(gpu):
    """Blocks whose bytes lie beyond 4 GiB from the layer's first: what is appended, seen and moved there."""
    import torch
    g = W.Geometry(1, 8, 128, 16, "bf16", 150000)
    raw = torch.empty(g.pool_bytes, dtype=torch.uint8, device=gpu)
    arena = torch.empty(g.S, dtype=torch.uint8, device=gpu)
    kp = kv.KVPool(g, raw, arena, flags=kv.KV_STAGING_DEVICE)
    b = kv.KVBatch(kp)
    view = raw.view(torch.bfloat16).view(1, 2, g.N, g.B, g.H, g.D)
    rng = np.random.default_rng(0)
    rows = [np.array([149999, 3, 149998, 140000, 139999], np.int32), np.array([131072, 131071, 149000], np.int32)]
    lens, q_lens, G = [77, 40], [20, 9], 4
    every = torch.from_numpy(np.concatenate(rows)).long().to(gpu)
    view[0, :, every] = torch.randn(2, 8, g.B, g.H, g.D, device=gpu).bfloat16()
    trees = [_parents(rng, n, "random") for n in q_lens]
    parents = torch.tensor(sum(trees, []), dtype=torch.int32, device=gpu)
    o, ids = R.csr(rows)
    kv.kv_check(b.set_trees(o, ids, lens, q_lens, G * 8, parents))
    k, v = (torch.randn(29, 8, 128, device=gpu).bfloat16() for _ in range(2))
    kv.kv_check(b.append(0, None, k, v))
    q = torch.randn(29, G * 8, 128, device=gpu).bfloat16()
    out = torch.empty_like(q)
    kv.kv_check(b.attn(0, q, out, 128 ** -0.5))
    small = view[0][:, every].double().cpu().numpy()
    at = [np.arange(5), np.arange(5, 8)]
    ref, tol, *_ = TR.attention(small, at, lens, q_lens, trees, q.double().cpu().numpy(), 128 ** -0.5, "bf16", 16)
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()
    tokens, chosen = _answers(rng, trees, q_lens, [5, 4])
    dev = lambda x: torch.from_numpy(x.astype(np.int32)).to(gpu)  # noqa: E731
    count, nxt, path = dev(np.zeros(2)), dev(np.zeros(2)), dev(np.zeros((2, 20)))
    kv.kv_check(b.accept(0, 1, dev(tokens), dev(chosen), count, path, nxt))
    after = view[0][:, every].double().cpu().numpy()
    t = 0
    for i, (tree, n, new) in enumerate(zip(trees, lens, q_lens)):
        way, follows = TR.accepted(tree, tokens[t:t + new], chosen[t:t + new])
        t += new
        assert count[i] == len(way) > 1 and nxt[i] == follows
        x = np.concatenate([np.arange(n - new), n - new + np.array(way)])
        y = np.arange(n - new + len(way))
        assert np.array_equal(after[:, at[i][y // 16], y % 16], small[:, at[i][x // 16], x % 16])


def test_a_chain_is_a_prompt(gpu):
    """A tree without a branch sees what the same tokens see that simply follow one another."""
    import torch
    H, D, B, G, lens, q_lens = 2, 128, 16, 4, [300, 77, 90], [40, 3, 1]
    p = Pool(gpu, W.Geometry(1, H, D, B, "bf16", 40), seed=2)
    rows = _tables(p.rng, 40, lens, B)
    p.fill(rows, lens)
    o, ids = R.csr(rows)
    q = torch.randn(44, G * H, D, device=gpu).bfloat16()
    ref, tol, *_ = R.attention(p.values()[0], rows, lens, q_lens, q.double().cpu().numpy(), D ** -0.5, "bf16", B)
    chain = torch.tensor([x for n in q_lens for x in _parents(p.rng, n, "chain")], dtype=torch.int32, device=gpu)
    out = torch.empty_like(q)
    kv.kv_check(p.batch.set_trees(o, ids, lens, q_lens, G * H, chain))
    kv.kv_check(p.batch.attn(0, q, out, D ** -0.5))
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()
    # and the batch forgets its trees when it is set again
    kv.kv_check(p.batch.set(o, ids, lens, q_lens, G * H))
    kv.kv_check(p.batch.attn(0, q, out, D ** -0.5))
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()


@pytest.mark.parametrize("what", ["nan", "inf", "two infs"])
@pytest.mark.parametrize("shape", [(2, 128, 16, 4), (2, 72, 5, 3), (1, 64, 16, 8), (1, 256, 32, 4), (2, 192, 4, 2)])
@pytest.mark.parametrize("new", [4, 30])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8_e4m3"])
def test_rows_feel_what_they_see_only(gpu, dtype, new, shape, what):
    """Values of drafted tokens that are not finite reach their own descendants' outputs, and no others'."""
    import torch
    if dtype == "fp8_e4m3" and what != "nan":
        pytest.skip("the type has no infinity")
    H, D, B, G = shape
    n = 170
    N = -(-n // B) + 2
    p = Pool(gpu, W.Geometry(1, H, D, B, dtype, N), seed=6)
    rows = _tables(p.rng, N, [n], B)
    p.fill(rows, [n])
    io_name = "f16" if dtype == "f16" else "bf16"
    parents = _parents(p.rng, new, "random")
    q = torch.from_numpy(p.rng.standard_normal((new, G * H, D))).to(_torch_type(io_name)).to(gpu)
    ref, tol, *_ = TR.attention(p.values()[0], rows, [n], [new], [parents], q.double().cpu().numpy(), D ** -0.5, io_name, B)
    inf = {"bf16": 0x7F80, "f16": 0x7C00, "fp8_e4m3": 0x7F}[dtype]
    nan = {"bf16": 0x7FC0, "f16": 0x7E00, "fp8_e4m3": 0x7F}[dtype]
    # (new token or None: the first cached one, element of its value, bits)
    bad = [(new // 2, 1, nan if what == "nan" else inf), (new - 2, 3, nan if what == "nan" else inf - 0x8000)]
    if what == "two infs":
        bad += [(1, 5, inf), (2, 5, inf - 0x8000)]
    if new == 30:
        bad.append((None, 7, nan if what == "nan" else inf))
    for j, d, b in bad:
        x = 0 if j is None else n - new + j
        p.bits()[0, 1, int(rows[0][x // B]), x % B, :, d] = b
    o, ids = R.csr(rows)
    out = torch.empty_like(q)
    kv.kv_check(p.batch.set_trees(o, ids, [n], [new], G * H, torch.tensor(parents, dtype=torch.int32, device=gpu)))
    kv.kv_check(p.batch.attn(0, q, out, D ** -0.5))
    got = out.double().cpu().numpy()
    _, family = TR.ancestry(parents)
    for j in range(new):
        special = {}
        for k, d, b in bad:
            if k is None or family[j, k]:
                special.setdefault(d, set()).add("nan" if b == nan else "+" if b == inf else "-")
        for d in range(D):
            if d not in special:
                assert (np.abs(got[j, :, d] - ref[j, :, d]) <= tol[j, :, d]).all(), (j, d)
            elif "nan" in special[d] or len(special[d]) > 1:
                assert np.isnan(got[j, :, d]).all(), (j, d)
            else:
                assert (got[j, :, d] == (np.inf if "+" in special[d] else -np.inf)).all(), (j, d)


def test_positions_follow_the_depth(gpu):
    """kv_append without positions turns drafted tokens by what is in front of them in their tree."""
    import torch
    H, D, B, G, lens, q_lens = 2, 64, 16, 2, [50, 33, 20, 0], [12, 5, 4, 1]
    p = Pool(gpu, W.Geometry(1, H, D, B, "bf16", 20), seed=3)
    rows = _tables(p.rng, 20, lens, B)
    p.fill(rows, lens)
    o, ids = R.csr(rows)
    trees = [_parents(p.rng, 12, "padded"), _parents(p.rng, 5, "strange"), None, [TR.ROOT]]
    every = [x for t, n in zip(trees, q_lens) for x in (t or [0] * n)]
    where = np.concatenate([n - k + (TR.depth(t) if t else np.arange(k)) if n else [0] for t, n, k in zip(trees, lens, q_lens)])
    kv.kv_check(p.batch.set_trees(o, ids, lens, q_lens, G * H, torch.tensor(every, dtype=torch.int64).to(torch.int32).to(gpu), [True, True, False, True]))
    turns = torch.from_numpy(kv.kv_rope_freqs(D)[1]).to(gpu)
    T = sum(q_lens)
    q, k, v = (torch.randn(T, h, D, device=gpu).bfloat16() for h in (G * H, H, H))
    got, want = torch.empty_like(q), torch.empty_like(q)
    kv.kv_check(p.batch.append(0, q, k, v, got, turns=turns))
    stored = p.bits().clone()
    kv.kv_check(p.batch.append(0, q, k, v, want, turns=turns, positions=torch.from_numpy(where.astype(np.int32)).to(gpu)))
    assert torch.equal(got, want) and torch.equal(stored, p.bits())


# name: geometry, lens, q_lens, kinds, length of the path that is planted, layers
ACCEPT = {
    "one row": ((1, 1, 64, 16, "bf16", False), [1], [1], ["chain"], [1]),
    "no path": ((1, 2, 64, 16, "bf16", False), [0, 9, 30, 40], [1, 0, 7, 5], ["chain", "chain", "none", "last alone"], [0, 0, 0, 0]),
    "trees and others": ((3, 2, 128, 16, "bf16", False), [100, 60, 77, 41], [12, 20, 30, 1], ["random", "-", "padded", "chain"], [5, 0, 4, 1]),
    "whole chains": ((2, 2, 64, 4, "f16", False), [90, 1024], [33, 1024], ["chain", "chain"], [33, 1024]),
    "odd heads": ((2, 3, 72, 5, "bf16", False), [90, 55, 64], [30, 7, 64], ["random", "random", "random"], [6, 3, 9]),
    "rows of 8 bytes": ((2, 1, 8, 2, "fp8_e4m3", False), [90, 55], [30, 7], ["random", "random"], [6, 3]),
    "rows of two workgroups": ((2, 40, 128, 16, "bf16", False), [90, 55], [30, 17], ["random", "random"], [6, 4]),
    "rows of many workgroups": ((1, 71, 256, 2, "f16", False), [40, 25], [30, 17], ["random", "random"], [6, 4]),
    "blocks of one": ((2, 2, 96, 1, "f16", False), [90, 155], [30, 100], ["random", "strange"], [6, 12]),
    "large trees": ((2, 2, 128, 16, "bf16", False), [1500, 1024], [1000, 1024], ["random", "random"], [160, 170]),
    "star": ((2, 2, 128, 16, "bf16", False), [600, 300], [500, 200], ["star", "star"], [2, 2]),
    "fp8": ((2, 4, 128, 32, "fp8_e4m3", False), [90, 155], [30, 100], ["random", "random"], [6, 12]),
    "fp8 with scales": ((2, 4, 128, 8, "fp8_e4m3", True), [90, 155], [30, 100], ["random", "random"], [6, 12]),
    "fp8 with scales, odd": ((2, 3, 72, 6, "fp8_e4m3", True), [90, 155], [30, 100], ["random", "padded"], [6, 12]),
}


def _answers(rng, trees, q_lens, lengths):
    """Drafted tokens and the model's choices, which follow a path of that many rows where the tree has one.  Siblings may have the same token."""
    tokens, chosen = [], []
    for tree, q, k in zip(trees, q_lens, lengths):
        tok, cho = rng.integers(0, 50, q), rng.integers(0, 50, q)
        if tree is not None and q:
            inside, family = TR.ancestry(tree)
            at = family.sum(1)
            ends = [j for j in range(q) if inside[j] and at[j] == k and family[j, 0]]
            if ends:
                u = int(rng.choice(ends))
                while tree[u] >= 0:
                    cho[tree[u]] = tok[u]
                    u = tree[u]
        tokens.append(tok)
        chosen.append(cho)
    return np.concatenate(tokens), np.concatenate(chosen)


@pytest.mark.parametrize("with_weights", [False, True])
@pytest.mark.parametrize("layout", ["layer", "block"])
@pytest.mark.parametrize("name", list(ACCEPT))
def test_accept(gpu, name, layout, with_weights):
    import torch
    (L, H, D, B, dtype, scales), lens, q_lens, kinds, lengths = ACCEPT[name]
    N = sum(-(-n // B) for n in lens) + 3
    p = Pool(gpu, W.Geometry(L, H, D, B, dtype, N, scales=scales), layout, seed=len(name))
    rows = _tables(p.rng, N, lens, B)
    p.fill(rows, lens)
    trees = [None if k == "-" else _parents(p.rng, q, k)[:q] for k, q in zip(kinds, q_lens)]
    tokens, chosen = _answers(p.rng, trees, q_lens, lengths)
    every = [x for t, q in zip(trees, q_lens) for x in (t if t is not None else [0] * q)]
    dev = lambda x: torch.tensor(x, dtype=torch.int64).to(torch.int32).to(gpu)  # noqa: E731
    o, ids = R.csr(rows)
    kv.kv_check(p.batch.set_trees(o, ids, lens, q_lens, H, dev(every), [t is not None for t in trees]))
    n, most = len(lens), max([q for t, q in zip(trees, q_lens) if t is not None] + [1])
    count, nxt, path = dev([-5] * n), dev([-5] * n), torch.full((n, most + 2), -5, dtype=torch.int32, device=gpu)
    layer, layers = (1, L - 1) if L > 1 else (0, 1)
    weights = torch.rand(layers, n, H, max(lens) + 2, device=gpu) if with_weights else None
    wstart = weights.clone() if with_weights else None
    before, values, sbefore = p.bits().clone(), p.view.contiguous().cpu().float().numpy(), None if p.scale is None else p.scale.clone()
    kv.kv_check(p.batch.accept(layer, layers, dev(tokens), dev(chosen), count, path, nxt, weights=weights))
    torch.cuda.synchronize()
    want = before.clone()
    t = 0
    longest = 0
    for i, (tree, length, new) in enumerate(zip(trees, lens, q_lens)):
        tok, cho = tokens[t:t + new], chosen[t:t + new]
        t += new
        if tree is None:
            assert count[i] == new and nxt[i] == cho[-1] and (path[i] == -5).all()
            continue
        way, follows = TR.accepted(tree, tok, cho) if length else ([], -1)
        longest = max(longest, len(way))
        assert count[i] == len(way) and nxt[i] == follows, i
        if length:
            assert path[i, :new].tolist() == way + [-1] * (new - len(way))
        assert (path[i, new:] == -5).all()
        base = length - new
        for k, j in enumerate(way):
            if k == j:
                continue
            sb, sp, db, dp = int(rows[i][(base + j) // B]), (base + j) % B, int(rows[i][(base + k) // B]), (base + k) % B
            if scales:
                s = sbefore[layer:layer + layers].cpu().numpy()
                f = (s[:, :, sb] / s[:, :, db])[..., None]
                again = torch.from_numpy(np.clip(values[layer:layer + layers, :, sb, sp] * f, -448, 448)).to(torch.float8_e4m3fn).view(torch.uint8)
                want[layer:layer + layers, :, db, dp] = again.to(gpu) if sb != db else before[layer:layer + layers, :, sb, sp]
            else:
                want[layer:layer + layers, :, db, dp] = before[layer:layer + layers, :, sb, sp]
        if with_weights:
            expect = wstart[:, i].clone()
            expect[:, :, base:base + new] = 0
            if way:
                expect[:, :, base:base + len(way)] = wstart[:, i][:, :, torch.tensor(way, device=gpu) + base]
            assert torch.equal(weights[:, i], expect)
    assert torch.equal(p.bits(), want)
    assert p.scale is None or torch.equal(p.scale, sbefore)
    if name not in ("one row", "no path"):
        assert longest > 1, "the case accepts nothing"


def test_accept_without_trees_and_without_layers(gpu):
    """In a batch without trees all new tokens stay; without layers nothing moves."""
    import torch
    p = Pool(gpu, W.Geometry(2, 2, 64, 16, "bf16", 12), seed=4)
    lens, q_lens = [30, 20, 0, 9], [3, 1, 1, 0]
    rows = _tables(p.rng, 12, lens, 16)
    p.fill(rows, lens)
    o, ids = R.csr(rows)
    before = p.bits().clone()
    chosen = torch.tensor([10, 11, 12, 13, 14], dtype=torch.int32, device=gpu)
    count, nxt = torch.zeros(4, dtype=torch.int32, device=gpu), torch.zeros(4, dtype=torch.int32, device=gpu)
    kv.kv_check(p.batch.set(o, ids, lens, q_lens, 4))
    kv.kv_check(p.batch.accept(0, 2, None, chosen, count, None, nxt))
    assert count.tolist() == [3, 1, 0, 0] and nxt.tolist() == [12, 13, -1, -1] and torch.equal(p.bits(), before)
    kv.kv_check(p.batch.set_trees(o, ids, lens, q_lens, 4, torch.tensor([-1, 0, 0, -1, -1], dtype=torch.int32, device=gpu)))
    tokens, path = torch.tensor([7, 5, 10, 1, 1], dtype=torch.int32, device=gpu), torch.empty(4, 3, dtype=torch.int32, device=gpu)
    kv.kv_check(p.batch.accept(0, 0, tokens, chosen, count, path, nxt))
    assert count.tolist() == [2, 1, 0, 0] and nxt.tolist() == [12, 13, -1, -1] and path[0].tolist() == [0, 2, -1] and torch.equal(p.bits(), before)


# name: geometry, G (0: no queries), lens, q_lens, rot, interleaved, (pad, off), axes, order
AXES = {
    "one token": ((1, 1, 64, 16, "bf16", False), 1, [1], [1], 64, False, (0, 0), 3, "sections"),
    "one axis": ((1, 2, 64, 16, "bf16", False), 1, [40, 9], [3, 9], 64, False, (0, 0), 1, "sections"),
    "decode": ((2, 4, 64, 16, "f16", False), 2, [5, 16, 17, 0, 300], [1, 1, 1, 1, 1], 64, True, (0, 0), 2, "turns"),
    "images": ((1, 2, 128, 16, "bf16", False), 4, [200, 41], [200, 7], 128, False, (0, 0), 3, "sections"),
    "four axes, part of the head": ((1, 2, 80, 5, "f16", False), 3, [90, 33], [4, 33], 54, False, (0, 0), 4, "turns"),
    "part of the head, interleaved": ((1, 3, 72, 5, "bf16", False), 1, [90, 33], [4, 33], 30, True, (3, 5), 3, "turns"),
    "two elements": ((1, 1, 128, 1, "bf16", False), 2, [9], [3], 2, False, (0, 0), 2, "last"),
    "nothing turned": ((1, 1, 128, 1, "bf16", False), 2, [9], [3], 0, False, (0, 0), 2, "turns"),
    "no queries": ((1, 2, 112, 16, "f16", False), 0, [90, 33], [4, 33], 112, False, (1, 1), 3, "sections"),
    "d 256": ((1, 2, 256, 16, "f16", False), 2, [90, 33], [4, 33], 256, False, (0, 0), 4, "sections"),
    "d 256, interleaved": ((1, 2, 256, 16, "bf16", False), 2, [90, 33], [4, 33], 128, True, (8, 8), 3, "any"),
    "fp8": ((2, 2, 128, 32, "fp8_e4m3", False), 4, [50, 7], [9, 1], 128, False, (0, 0), 3, "any"),
    "fp8 with scales": ((2, 4, 128, 32, "fp8_e4m3", True), 2, [50, 70, 1], [40, 1, 1], 64, False, (0, 0), 3, "sections"),
    "fp8 with scales, strides of 2 bytes": ((2, 2, 96, 4, "fp8_e4m3", True), 2, [50, 70, 1], [40, 1, 1], 34, False, (1, 3), 2, "any"),
}


@pytest.mark.parametrize("name", list(AXES))
def test_append_axes(gpu, name):
    import torch
    (L, H, D, B, dtype, scales), G, lens, q_lens, rot, inter, (pad, off), axes, order = AXES[name]
    N = sum(-(-n // B) for n in lens) + 3
    p = Pool(gpu, W.Geometry(L, H, D, B, dtype, N, scales=scales), seed=len(name))
    rows = _tables(p.rng, N, lens, B)
    p.fill(rows, lens)
    layer, magnitude, pairs, T = L - 1, 1.25, rot // 2, sum(q_lens)
    freq = 500000.0 ** (-np.arange(pairs) * 2.0 / max(rot, 1)) / (2 * np.pi)
    turns = torch.from_numpy(np.array([int(round(f * 2.0 ** 64)) for f in freq], np.int64)).to(gpu) if rot else None
    pair_axes = {"turns": np.arange(pairs) % axes, "sections": np.arange(pairs) * axes // max(pairs, 1), "last": np.full(pairs, axes - 1),
                 "any": p.rng.integers(0, axes, pairs)}[order].astype(np.int32)
    pos = p.rng.integers(0, 3000, (axes, T))
    pos[:, T // 2] = p.rng.integers(2 ** 30, 2 ** 31, axes)  # far ones, too
    big = torch.full((axes, T + 3), -1, dtype=torch.int32, device=gpu)
    positions = big[:, :T]
    positions.copy_(torch.from_numpy(pos))
    index = np.concatenate([np.arange(n - q, n) if n else np.array([-1]) for n, q in zip(lens, q_lens)])
    req = np.repeat(np.arange(len(lens)), q_lens)
    o, ids = R.csr(rows)
    kv.kv_check(p.batch.set(o, ids, lens, q_lens, max(G, 1) * H))
    for io_name in ([dtype] if dtype != "fp8_e4m3" else ["bf16", "f16"]):
        io, u = _torch_type(io_name), R.U[io_name]
        new = lambda n: _heads(torch, gpu, p.rng.standard_normal((T, n, D)) * (1.0 if dtype != "fp8_e4m3" else 20.0), io, pad, off)  # noqa: E731
        q = new(G * H) if G else None
        k, v = new(H), new(H)
        q_out = _heads(torch, gpu, np.zeros((T, max(G, 1) * H, D)), io, pad, off) if G else None
        scale = [torch.from_numpy(p.rng.uniform(0.03, 0.06, H).astype(np.float32)).to(gpu) for _ in range(2)] if scales else [None, None]
        before = p.bits().clone()
        kv.kv_check(p.batch.append(layer, q, k, v, q_out, turns=turns, interleaved=inter, magnitude=magnitude, positions=positions, pair_axes=pair_axes,
                                   k_scale=scale[0], v_scale=scale[1]))
        torch.cuda.synchronize()
        slop = 2.0 ** -15  # of the products' magnitudes: what cosines, sines and the products in 32 bits may be off by
        if G:
            ref, mag = TR.rotate_axes(q.double().cpu().numpy(), pos, pair_axes, freq, magnitude, inter)
            assert (np.abs(q_out.double().cpu().numpy() - ref) <= u * np.abs(ref) + 2 * slop * mag + 2.0 ** -25).all()
        rk, mk = TR.rotate_axes(k.double().cpu().numpy(), pos, pair_axes, freq, magnitude, inter)
        rv = v.double().cpu().numpy()
        live = index >= 0
        blk = np.array([rows[r][x // B] if x >= 0 else 0 for r, x in zip(req, index)])[live].astype(np.int64)
        place = (index % B)[live]
        stored = p.view.contiguous().cpu().float().numpy().astype(np.float64)[layer]
        for c, ref, mag in ((0, rk, mk), (1, rv, np.abs(rv) * 0)):
            ref, mag, got = ref[live], mag[live], stored[c, blk, place]
            if dtype == "fp8_e4m3":
                if scales:
                    s = scale[c].double().cpu().numpy()[None, :, None]
                    ref, mag = ref / s, mag / s
                    assert torch.equal(p.scale[layer, c, torch.from_numpy(blk).to(gpu)], scale[c].expand(len(blk), H))
                ref = np.clip(ref, -448, 448)
                # half a step of e4m3 (2^-4 relative, 2^-10 below its normal range)
                assert (np.abs(got - ref) <= np.maximum(2.0 ** -4 * np.abs(ref), 2.0 ** -10) + 2 * slop * mag + 2.0 ** -20).all()
            else:
                assert (np.abs(got - ref) <= u * np.abs(ref) + 2 * slop * mag + 2.0 ** -25).all()
        # nothing else changes
        same = torch.ones(p.view.shape[:4], dtype=torch.bool, device=gpu)
        same[layer][:, torch.from_numpy(blk).to(gpu), torch.from_numpy(place).to(gpu)] = False
        assert torch.equal(p.bits()[same], before[same])


def test_one_position_on_all_axes_is_plain(gpu):
    """Text: the same bits as kv_append gives."""
    import torch
    p = Pool(gpu, W.Geometry(1, 2, 128, 16, "bf16", 12), seed=4)
    rows = _tables(p.rng, 12, [100], 16)
    p.fill(rows, [100])
    o, ids = R.csr(rows)
    kv.kv_check(p.batch.set(o, ids, [100], [60], 8))
    q, k, v = (torch.randn(60, h, 128, device=gpu).bfloat16() for h in (8, 2, 2))
    turns = torch.from_numpy(kv.kv_rope_freqs(128)[1]).to(gpu)
    where = torch.randint(0, 100000, (60,), dtype=torch.int32, device=gpu)
    a, b = torch.empty_like(q), torch.empty_like(q)
    kv.kv_check(p.batch.append(0, q, k, v, a, turns=turns, positions=where))
    stored = p.bits().clone()
    kv.kv_check(p.batch.append(0, q, k, v, b, turns=turns, positions=where.expand(3, 60).contiguous(), pair_axes=np.arange(64) % 3))
    assert torch.equal(a, b) and torch.equal(stored, p.bits())


def _step(p, gpu, rows, lens, q_lens, trees, Hq, stream=None):
    """One step's calls on a batch whose trees are set: append, attention in every layer, acceptance.  -> what is called, and its outputs"""
    import torch
    g, T, n = p.g, sum(q_lens), len(lens)
    gen = torch.Generator(device=gpu).manual_seed(1)
    rand = lambda h: torch.randn(T, h, g.D, device=gpu, generator=gen).bfloat16()  # noqa: E731
    qs, ks, vs = [[rand(h) for _ in range(g.L)] for h in (Hq, g.H, g.H)]
    turned, outs = [torch.empty_like(q) for q in qs], [torch.empty_like(q) for q in qs]
    tokens, chosen = _answers(p.rng, trees, q_lens, [4] * n)
    tokens, chosen = (torch.from_numpy(x.astype(np.int32)).to(gpu) for x in (tokens, chosen))
    count, nxt = torch.zeros(n, dtype=torch.int32, device=gpu), torch.zeros(n, dtype=torch.int32, device=gpu)
    path = torch.zeros(n, max(q_lens), dtype=torch.int32, device=gpu)
    turns = torch.from_numpy(kv.kv_rope_freqs(g.D)[1]).to(gpu)

    def call():
        for layer in range(g.L):
            kv.kv_check(p.batch.append(layer, qs[layer], ks[layer], vs[layer], turned[layer], turns=turns, stream=stream))
            kv.kv_check(p.batch.attn(layer, turned[layer], outs[layer], g.D ** -0.5, stream=stream))
        kv.kv_check(p.batch.accept(0, g.L, tokens, chosen, count, path, nxt, stream=stream))
    return call, lambda: [x.clone() for x in outs + [count, path, nxt, p.bits()]], (qs, ks, tokens, chosen)


def test_a_captured_step(gpu):
    """A step with drafts in a graph, replayed with new inputs between eager work of its own, gives what the calls give."""
    import torch
    lens, q_lens, Hq = [300, 77, 90, 600], [12, 5, 1, 40], 8
    p = Pool(gpu, W.Geometry(2, 2, 128, 16, "bf16", 80), seed=9)
    rows = _tables(p.rng, 80, lens, 16)
    p.fill(rows, lens)
    trees = [_parents(p.rng, q, "random") for q in q_lens]
    parents = torch.tensor(sum(trees, []), dtype=torch.int32, device=gpu)
    o, ids = R.csr(rows)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    call, outputs, (qs, ks, tokens, chosen) = _step(p, gpu, rows, lens, q_lens, trees, Hq, st)
    start = p.bits().clone()
    torch.cuda.synchronize()
    kv.kv_check(p.batch.set_trees(o, ids, lens, q_lens, Hq, parents, stream=st))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        call()
    torch.cuda.synchronize()
    for turn in range(4):
        for x in qs + ks:
            x.normal_()
        new_tokens, new_chosen = _answers(p.rng, trees, q_lens, [1 + turn] * 4)
        tokens.copy_(torch.from_numpy(new_tokens.astype(np.int32)))
        chosen.copy_(torch.from_numpy(new_chosen.astype(np.int32)))
        p.bits().copy_(start)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            call()
        st.synchronize()
        want = outputs()
        for _ in range(2):
            p.bits().copy_(start)
            torch.cuda.synchronize()
            with torch.cuda.stream(st):
                graph.replay()
            st.synchronize()
            got = outputs()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), turn


def test_parents_are_read_in_the_order_of_the_stream(gpu):
    """The drafts come from work that is still under way on the stream, and the tensor may be changed behind the call."""
    import torch
    lens, q_lens = [300, 77], [12, 20]
    p = Pool(gpu, W.Geometry(1, 2, 128, 16, "bf16", 40), seed=10)
    rows = _tables(p.rng, 40, lens, 16)
    p.fill(rows, lens)
    o, ids = R.csr(rows)
    trees = [_parents(p.rng, q, "random") for q in q_lens]
    good = torch.tensor(sum(trees, []), dtype=torch.int32, device=gpu)
    q = torch.randn(32, 8, 128, device=gpu).bfloat16()
    ref, tol, *_ = TR.attention(p.values()[0], rows, lens, q_lens, trees, q.double().cpu().numpy(), 0.1, "bf16", 16)
    st, other = torch.cuda.Stream(), torch.cuda.Stream()
    parents, out = torch.full_like(good, -2), torch.zeros_like(q)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        torch.cuda._sleep(2_000_000)
        parents.copy_(good)
        kv.kv_check(p.batch.set_trees(o, ids, lens, q_lens, 8, parents))
        parents.fill_(-2)
    with torch.cuda.stream(other):  # (the batch orders its own work between streams)
        kv.kv_check(p.batch.attn(0, q, out, 0.1))
    torch.cuda.synchronize()
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()


def test_two_batches_at_once(gpu):
    """Two batches on one pool, on streams of their own, do not share anything."""
    import torch
    p = Pool(gpu, W.Geometry(1, 2, 128, 16, "bf16", 140), seed=12)
    lens, q_lens = [[900, 77], [500, 600]], [[12, 20], [33, 9]]
    every = _tables(p.rng, 140, lens[0] + lens[1], 16)
    rows = [every[:2], every[2:]]
    p.fill(every, lens[0] + lens[1])
    batches, streams = [p.batch, kv.KVBatch(p.kp)], [torch.cuda.Stream(), torch.cuda.Stream()]
    work = []
    for b, r, n, ql in zip(batches, rows, lens, q_lens):
        trees = [_parents(p.rng, q, "random") for q in ql]
        q = torch.randn(sum(ql), 8, 128, device=gpu).bfloat16()
        ref, tol, *_ = TR.attention(p.values()[0], r, n, ql, trees, q.double().cpu().numpy(), 0.1, "bf16", 16)
        work.append((b, R.csr(r), n, ql, torch.tensor(sum(trees, []), dtype=torch.int32, device=gpu), q, torch.empty_like(q), ref, tol))
    torch.cuda.synchronize()
    for turn in range(3):
        for st, (b, (o, ids), n, ql, parents, q, out, _, _) in zip(streams, work):
            with torch.cuda.stream(st):
                out.zero_()
                kv.kv_check(b.set_trees(o, ids, n, ql, 8, parents))
                kv.kv_check(b.attn(0, q, out, 0.1))
        torch.cuda.synchronize()
        for *_, out, ref, tol in work:
            assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()


def test_the_same_bits_twice(gpu):
    import torch
    p, rows, trees, parents = _drafts(gpu, "many behind a prefix")
    (L, H, D, B, *_), G, lens, q_lens = TREES["many behind a prefix"][:4]
    o, ids = R.csr(rows)
    q = torch.randn(sum(q_lens), G * H, D, device=gpu).bfloat16()
    kv.kv_check(p.batch.set_trees(o, ids, lens, q_lens, G * H, parents, [t is not None for t in trees]))
    got = []
    for _ in range(3):
        out, lse, w = torch.empty_like(q), torch.empty(q.shape[:2], device=gpu), torch.zeros(len(lens), H, max(lens), device=gpu)
        kv.kv_check(p.batch.attn(0, q, out, D ** -0.5, lse=lse, weights=w))
        got.append((out.view(torch.int16), lse.view(torch.int32), w.view(torch.int32)))
    for x in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(x, got[0]))


def test_the_drafting_example(gpu):
    """Prompts with images, drafts, attention over their trees, and accepted paths in one loop: what it leaves in the cache and answers is what the same
    tokens give one at a time, 16-bit roundings apart."""
    from paper_2510_02758_amd import stream_demo
    r = stream_demo.speculate()
    assert r["accepted"] > 1 and r["tokens"] >= 20
    assert r["hidden"] < 0.05 and r["cache"] < 0.05
