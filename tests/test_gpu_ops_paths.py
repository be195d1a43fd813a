"""The attention's ways through its kernels that only larger batches take (ops_paths.py), on a real MI355X, against the definition in 64 bits.  The
reference runs on the GPU: plain products, exponentials and sums in 64 bits, with the bounds that ops_ref.py derives."""
import numpy as np
import pytest

import ops_ref as R
from ops_paths import PATHS, tables
from paper_2510_02758_amd import kvswap as kv
from paper_2510_02758_amd import workloads as W

pytestmark = pytest.mark.gpu


class _Batch:
    """A pool of random values with NaN wherever no request has a token, and a batch on it."""

    def __init__(self, gpu, name):
        import torch
        (H, D, B, dtype, scales), self.G, self.lens, self.q_lens, shared, _ = PATHS[name]
        self.H, self.D, self.B, self.dtype = H, D, B, dtype
        N = sum(-(-n // B) for n in self.lens) + 3
        g = W.Geometry(1, H, D, B, dtype, N, scales=scales)
        self.rows = tables(np.random.default_rng(len(name)), N, self.lens, B, shared)
        gen = torch.Generator(device=gpu).manual_seed(len(name))
        fp8 = dtype == "fp8_e4m3"
        stored = {"f16": torch.float16, "bf16": torch.bfloat16, "fp8_e4m3": torch.float8_e4m3fn}[dtype]
        x = (torch.randn(2, N, B, H, D, generator=gen, device=gpu) * (30.0 if fp8 else 1.0)).to(stored)
        used = torch.zeros(N * B, dtype=torch.bool, device=gpu)
        self.at = []
        for row, n in zip(self.rows, self.lens):
            i = torch.arange(n, device=gpu)
            self.at.append(torch.from_numpy(row.astype(np.int64)).to(gpu)[i // B] * B + i % B if n else i)
            used[self.at[-1]] = True
        bits = x.view(torch.uint8 if fp8 else torch.int16)
        bits[:, ~used.view(N, B)] = {"fp8_e4m3": 0x7F, "bf16": 0x7FC1, "f16": 0x7E01}[dtype]
        self.raw = bits.view(torch.uint8).reshape(-1).contiguous()
        self.values = x.view(stored).view(2, N * B, H, D)
        self.scale = torch.empty(2, N, H, device=gpu).uniform_(0.01, 0.05, generator=gen) if scales else None
        self.arena = torch.empty(g.S, dtype=torch.uint8, device=gpu)
        self.kp = kv.KVPool(g, self.raw, self.arena, scale=None if self.scale is None else self.scale.view(torch.uint8).view(-1), flags=kv.KV_STAGING_DEVICE)
        self.batch = kv.KVBatch(self.kp)
        self.T = sum(self.q_lens)
        self.q = lambda io: torch.randn(self.T, H * self.G, D, generator=gen, device=gpu).to(io)

    def kv(self, i, h):
        """Keys and values [length, D] of request i and head h in 64 bits."""
        import torch
        x = self.values[:, :, h].view(torch.uint8 if self.dtype == "fp8_e4m3" else self.values.dtype)[:, self.at[i]].view(self.values.dtype).double()
        if self.scale is not None:
            x = x * self.scale[:, self.at[i] // self.B, h].double()[..., None]
        return x

    def expected(self, q, scale, u):
        import torch
        H, G, D, T = self.H, self.G, self.D, self.T
        q = q.double().view(T, H, G, D)
        out, tol = torch.zeros_like(q), torch.zeros_like(q)
        lse, ltol = q.new_full((T, H, G), -torch.inf), q.new_zeros(T, H, G)
        weights, wtol = [], []
        t = 0
        for i, (n, new) in enumerate(zip(self.lens, self.q_lens)):
            weights.append(q.new_zeros(H, n))
            wtol.append(q.new_zeros(H, n))
            if n and new:
                hidden = torch.ones(new, n, dtype=torch.bool, device=q.device).triu(n - new + 1).repeat_interleave(G, 0)
                for h in range(H):
                    k, v = self.kv(i, h)
                    rows = q[t:t + new, h].reshape(new * G, D)
                    z = (rows @ k.t().contiguous() * scale).masked_fill_(hidden, -torch.inf)
                    size = (rows.abs() @ k.abs().t().contiguous()).masked_fill_(hidden, 0.0).amax(-1) * abs(scale)
                    ds = (D + 4) * 2.0 ** -23 * size + 2.0 ** -22 * z.masked_fill(hidden, 0.0).abs().amax(-1) + 2.0 ** -20
                    l = z.logsumexp(-1)
                    p = (z - l[:, None]).exp()
                    o, spread = p @ v, p @ v.abs()
                    seen = (~hidden).sum(-1)
                    # (f16 has no numbers between 0 and 2^-24)
                    bound = u * o.abs() + spread * (u + 2 * ds + (seen + 64) * 2.0 ** -23)[:, None] + (2.0 ** -25 if u < 2.0 ** -8 else 1e-30)
                    out[t:t + new, h], tol[t:t + new, h] = o.view(new, G, D), bound.view(new, G, D)
                    lse[t:t + new, h], ltol[t:t + new, h] = l.view(new, G), (2 * ds + 2.0 ** -22 * (1 + l.abs())).view(new, G)
                    weights[i][h] = p.sum(0)
                    wtol[i][h] = (p * (4 * ds + 2.0 ** -20)[:, None]).sum(0)
            t += new
        return out.view(T, H * G, D), tol.view(T, H * G, D), lse.view(T, H * G), ltol.view(T, H * G), weights, wtol


@pytest.mark.parametrize("name", list(PATHS))
def test_attention_of_large_batches(gpu, name):
    import torch
    b = _Batch(gpu, name)
    o, ids = R.csr(b.rows)
    kv.kv_check(b.batch.set(o, ids, b.lens, b.q_lens, b.H * b.G))
    scale = 1.5 * b.D ** -0.5
    for io_name in ([b.dtype] if b.dtype != "fp8_e4m3" else ["bf16", "f16"]):
        q = b.q({"bf16": torch.bfloat16, "f16": torch.float16}[io_name])
        ref, tol, rlse, ltol, rw, wtol = b.expected(q, scale, R.U[io_name])
        before = torch.rand(len(b.lens), b.H, max(b.lens) + 3, device=gpu) * 2
        for weights in (None, before.clone()):
            out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=gpu)
            kv.kv_check(b.batch.attn(0, q, out, scale, lse=lse, weights=weights))
            torch.cuda.synchronize()
            assert bool(((out.double() - ref).abs() <= tol).all()), float(((out.double() - ref).abs() / tol).nan_to_num(1e9).max())
            none = rlse.isinf()
            assert torch.equal(lse.isinf(), none) and bool(((lse.double() - rlse).abs() <= ltol)[~none].all())
            if weights is None:
                continue
            for i, n in enumerate(b.lens):
                want = before[i].double()
                want[:, :n] += rw[i]
                assert bool(((weights[i].double() - want)[:, :n].abs() <= wtol[i] + 2.0 ** -22 * want[:, :n].abs() + 1e-30).all()), i
                assert torch.equal(weights[i, :, n:], before[i, :, n:]), i


@pytest.mark.parametrize("name", ["four heads a workgroup", "four heads a workgroup, fp8", "many prefixes", "a long prefix", "very many pieces", "a long prompt",
                                  "more query heads than rows, a prefix"])
def test_first_weights_in_a_capture(gpu, name):
    """A batch whose first call with weights is in a capture has no room for products: they are computed again, in every replay.  The same batch
    with room gives the same weights, by another sum."""
    import torch
    b = _Batch(gpu, name)
    o, ids = R.csr(b.rows)
    st = torch.cuda.Stream()
    io_name = "f16" if b.dtype == "f16" else "bf16"
    q = b.q({"bf16": torch.bfloat16, "f16": torch.float16}[io_name])
    scale = 1.5 * b.D ** -0.5
    out, weights = torch.empty_like(q), torch.zeros(len(b.lens), b.H, max(b.lens), device=gpu)
    torch.cuda.synchronize()
    kv.kv_check(b.batch.set(o, ids, b.lens, b.q_lens, b.H * b.G, stream=st))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        kv.kv_check(b.batch.attn(0, q, out, scale, weights=weights, stream=st))
    for turn in range(3):
        if turn:
            q.copy_(b.q(q.dtype))
        ref, tol, _, _, rw, wtol = b.expected(q, scale, R.U[io_name])
        out.zero_()
        weights.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert bool(((out.double() - ref).abs() <= tol).all()), turn
        for i, n in enumerate(b.lens):
            assert bool(((weights[i, :, :n].double() - rw[i]).abs() <= wtol[i] + 2.0 ** -22 * rw[i] + 1e-30).all()), (turn, i)
        again = torch.zeros_like(weights)
        torch.cuda.synchronize()
        kv.kv_check(b.batch.attn(0, q, out, scale, weights=again, stream=st))
        torch.cuda.synchronize()
        for i, n in enumerate(b.lens):
            assert bool(((again[i, :, :n].double() - rw[i]).abs() <= wtol[i] + 2.0 ** -22 * rw[i] + 1e-30).all()), (turn, i)
