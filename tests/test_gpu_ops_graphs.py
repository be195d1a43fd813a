"""Captured calls of the operators on the pool's contents, replayed on streams of their own."""
import numpy as np
import pytest

import ops_ref as R
from paper_2510_02758_amd import kvswap as kv
from paper_2510_02758_amd import workloads as W
from test_gpu_ops import Pool, _tables

pytestmark = pytest.mark.gpu


def _long_batch(gpu):
    H, D, B, G, lens = 2, 128, 16, 4, [20011, 300]
    N = sum(-(-n // B) for n in lens) + 3
    p = Pool(gpu, W.Geometry(1, H, D, B, "bf16", N), seed=13)
    rows = _tables(p.rng, N, lens, B)
    p.fill(rows, lens)
    return p, rows, lens, G * H, D


def test_a_new_batch_comes_after_replays_on_another_stream(gpu):
    """Replays that are under way go on with the tables they were captured with; the new batch and its calls come after them."""
    import torch
    p, rows, lens, Hq, D = _long_batch(gpu)
    order = ([0, 1], [1, 0])
    csr = [R.csr([rows[i] for i in o]) + ([lens[i] for i in o],) for o in order]
    q = torch.randn(2, Hq, D, device=gpu).bfloat16()
    want = []
    for o, ids, n in csr:
        out, w = torch.empty_like(q), torch.zeros(2, p.g.H, max(lens), device=gpu)
        kv.kv_check(p.batch.set(o, ids, n, [1, 1], Hq))
        kv.kv_check(p.batch.attn(0, q, out, D ** -0.5, weights=w))
        torch.cuda.synchronize()
        want.append((out, w))
    st, other = torch.cuda.Stream(), torch.cuda.Stream()
    for turn in range(3):
        outs, ws = [torch.zeros_like(q) for _ in range(2)], [torch.zeros_like(want[0][1]) for _ in range(2)]
        torch.cuda.synchronize()
        o, ids, n = csr[0]
        kv.kv_check(p.batch.set(o, ids, n, [1, 1], Hq, stream=st))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            kv.kv_check(p.batch.attn(0, q, outs[0], D ** -0.5, stream=st))
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            for _ in range(20):
                graph.replay()
        o, ids, n = csr[1]
        kv.kv_check(p.batch.set(o, ids, n, [1, 1], Hq, stream=st))
        kv.kv_check(p.batch.attn(0, q, outs[1], D ** -0.5, weights=ws[1], stream=st))
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0][0]) and torch.equal(outs[1], want[1][0]) and torch.equal(ws[1], want[1][1]), turn
