"""The operators on the pool's contents (rotary append, attention, eviction) on a real MI355X, against plain implementations in 64 bits
(ops_ref.py)."""
import numpy as np
import pytest

import ops_ref as R
from paper_2510_02758_amd import kvswap as kv
from paper_2510_02758_amd import workloads as W

pytestmark = pytest.mark.gpu


def _torch_type(dtype):
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16, "fp8_e4m3": torch.float8_e4m3fn}[dtype]


class Pool:
    """A pool with values, and its float64 picture.  Every place that no request's token has holds a NaN."""

    def __init__(self, gpu, g, layout="layer", seed=0, size=1.0):
        import torch
        self.g, self.torch, self.gpu, self.layout = g, torch, gpu, layout
        self.rng = np.random.default_rng(seed)
        self.raw = torch.zeros(g.pool_bytes, dtype=torch.uint8, device=gpu)
        t = self.raw.view(_torch_type(g.dtype))
        if layout == "layer":
            self.view = t.view(g.L, 2, g.N, g.B, g.H, g.D)
        else:
            self.view = t.view(g.N, g.L, 2, g.B, g.H, g.D).permute(1, 2, 0, 3, 4, 5)
        self.scale = None
        if g.scales:
            self.scale = torch.from_numpy(self.rng.uniform(0.01, 0.05, (g.L, 2, g.N, g.H)).astype(np.float32)).to(gpu)
        self.size = size
        arena = torch.empty(g.S, dtype=torch.uint8, device=gpu)
        self.kp = kv.KVPool(g, self.raw, arena, scale=None if self.scale is None else self.scale.view(torch.uint8).view(-1),
                            strides=None if layout == "layer" else g.strides_block_major, flags=kv.KV_STAGING_DEVICE)
        self.batch = kv.KVBatch(self.kp)

    def fill(self, tables, lens):
        """Random values where the requests have tokens, NaN in all other places."""
        g, torch = self.g, self.torch
        used = np.zeros((g.N, g.B), bool)
        for row, n in zip(tables, lens):
            x = np.arange(n)
            used[np.asarray(row, np.int64)[x // g.B], x % g.B] = True
        vals = self.rng.standard_normal((g.L, 2, g.N, g.B, g.H, g.D)).astype(np.float32) * (30.0 if g.dtype == "fp8_e4m3" else self.size)
        x = torch.from_numpy(vals).to(_torch_type(g.dtype))
        bits = x.view(torch.uint8 if g.dtype == "fp8_e4m3" else torch.int16)
        nan = {"fp8_e4m3": 0x7F, "bf16": 0x7FC1, "f16": 0x7E01}[g.dtype]
        bits[:, :, torch.from_numpy(~used)] = nan
        self.write(bits)

    def write(self, bits):
        self.bits().copy_(bits.to(self.gpu))

    def bits(self):
        return self.view.view(self.torch.uint8 if self.g.dtype == "fp8_e4m3" else self.torch.int16)

    def values(self):
        x = self.view.contiguous().cpu().float().numpy().astype(np.float64)
        if self.scale is not None:
            x = x * self.scale.cpu().numpy().astype(np.float64)[:, :, :, None, :, None]
        return x


def _tables(rng, N, lens, B, shared=()):
    """Tables of distinct blocks; shared: (request, of which request, blocks) begins with the other's first blocks."""
    perm, at, rows = rng.permutation(N).astype(np.int32), 0, []
    for n in lens:
        need = -(-n // B)
        rows.append(perm[at:at + need].copy())
        at += need
    for i, of, k in shared:
        assert k <= len(rows[i]) and k <= len(rows[of])
        rows[i][:k] = rows[of][:k]
    return rows


def _heads(torch, gpu, x, io, pad=0, off=0):
    """x [T, heads, D] as a device tensor inside a larger one, `off` elements in and with `pad` behind each head."""
    T, n, D = x.shape
    big = torch.full((off + T * (n * (D + pad) + pad) + 64,), float("nan"), dtype=io, device=gpu)
    v = big[off:].as_strided((T, n, D), (n * (D + pad) + pad, D + pad, 1), off)
    v.copy_(torch.from_numpy(x).to(io))
    return v


# name: geometry (L, H, D, B, dtype, scales), G, lens, q_lens, shared, layout, (pad, off)
ATTN = {
    "one token": ((1, 1, 64, 16, "bf16", False), 1, [1], [1], (), "layer", (0, 0)),
    "nothing cached": ((2, 2, 64, 16, "f16", False), 2, [0, 0], [1, 1], (), "layer", (0, 0)),
    "short and empty": ((2, 4, 64, 16, "f16", False), 2, [0, 1, 15, 16, 17, 31, 32, 33, 127, 128, 129], [1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1], (), "layer", (0, 0)),
    "requests without a row": ((1, 2, 128, 16, "bf16", False), 4, [40, 100, 7], [0, 1, 0], (), "layer", (0, 0)),
    "odd heads": ((2, 3, 72, 5, "bf16", False), 5, [3, 77, 200], [1, 1, 1], (), "layer", (8, 8)),
    "d 80, strides of 2 bytes": ((1, 2, 80, 16, "f16", False), 3, [90, 333], [1, 2], (), "block", (3, 5)),
    "d 96": ((1, 2, 96, 1, "bf16", False), 7, [300, 2], [1, 1], (), "layer", (0, 0)),
    "d 112": ((1, 2, 112, 4, "f16", False), 16, [130, 65], [3, 1], (), "block", (0, 0)),
    "d 192": ((1, 2, 192, 16, "bf16", False), 2, [400, 31], [1, 4], (), "layer", (0, 0)),
    "d 256": ((1, 1, 256, 20, "f16", False), 8, [500, 41], [2, 1], (), "layer", (0, 0)),
    "d 256, blocks of 16": ((2, 2, 256, 16, "bf16", False), 4, [300, 37], [1, 1], (), "layer", (0, 0)),
    "d 64, blocks of 32": ((2, 3, 64, 32, "bf16", False), 16, [1300, 37, 128], [1, 1, 1], (), "block", (0, 0)),
    "fp8 d 64, blocks of 16": ((2, 3, 64, 16, "fp8_e4m3", True), 5, [1300, 37, 128], [1, 1, 1], (), "block", (0, 0)),
    "fp8 d 256, blocks of 48": ((2, 2, 256, 48, "fp8_e4m3", True), 3, [700, 37, 128], [1, 1, 1], (), "layer", (0, 0)),
    "d 8": ((1, 2, 8, 8, "bf16", False), 2, [70], [1], (), "layer", (0, 0)),
    "many query heads": ((1, 1, 128, 16, "bf16", False), 71, [290, 45], [1, 2], (), "layer", (0, 0)),
    "long, few rows": ((1, 1, 128, 16, "bf16", False), 8, [20011], [1], (), "layer", (0, 0)),
    "long, token by token": ((1, 1, 64, 1, "f16", False), 4, [9001], [1], (), "layer", (0, 0)),
    "fp8": ((2, 2, 128, 32, "fp8_e4m3", False), 4, [50, 700], [1, 1], (), "layer", (0, 0)),
    "fp8 with scales": ((2, 4, 128, 32, "fp8_e4m3", True), 1, [257, 64, 1000], [1, 1, 1], (), "layer", (0, 0)),
    "fp8 with scales, odd": ((2, 2, 72, 6, "fp8_e4m3", True), 3, [257, 64, 5], [1, 3, 2], (), "layer", (1, 1)),
    "fp8 with scales, d 64": ((2, 2, 64, 4, "fp8_e4m3", True), 9, [100, 511], [2, 1], (), "block", (0, 0)),
    "fp8 d 256": ((2, 1, 256, 16, "fp8_e4m3", True), 4, [100, 511], [40, 1], (), "layer", (0, 0)),
    "prompt from nothing": ((1, 2, 128, 16, "bf16", False), 4, [150], [150], (), "layer", (0, 0)),
    "prompt chunks": ((1, 2, 128, 16, "bf16", False), 4, [600, 70, 333], [130, 70, 1], (), "layer", (0, 0)),
    "prompt chunk, d 64, blocks of 16": ((1, 3, 64, 16, "f16", False), 2, [600, 300], [290, 77], (), "block", (0, 0)),
    "prompt chunk, d 256, blocks of 32": ((1, 1, 256, 32, "bf16", False), 3, [600, 300], [290, 77], (), "layer", (8, 8)),
    "prompt chunk, d 64": ((1, 3, 64, 5, "f16", False), 1, [600, 300], [290, 77], (), "layer", (5, 3)),
    "prompt chunk, fp8": ((2, 2, 128, 16, "fp8_e4m3", True), 2, [500, 91], [200, 30], (), "layer", (0, 0)),
    "prompt chunk, d 192": ((1, 1, 192, 16, "bf16", False), 3, [420, 90], [170, 64], (), "layer", (0, 0)),
    "prompt chunk, d 256": ((1, 1, 256, 16, "f16", False), 6, [300], [140], (), "layer", (0, 0)),
    "a shared prefix": ((1, 2, 128, 16, "bf16", False), 4, [330, 340, 350, 360, 400], [1] * 5, ((1, 0, 20), (2, 0, 20), (3, 0, 20), (4, 0, 20)), "layer", (0, 0)),
    "a tree of prefixes": ((1, 2, 64, 16, "f16", False), 2, [400, 400, 410, 500, 90, 33], [1, 2, 1, 3, 1, 1],
                           ((1, 0, 24), (2, 0, 24), (3, 1, 16), (4, 0, 5), (5, 4, 2)), "layer", (0, 0)),
    "a shared prefix and nothing else": ((1, 2, 128, 16, "bf16", False), 2, [320, 320, 320], [1, 1, 1], ((1, 0, 20), (2, 0, 20)), "layer", (0, 0)),
    "many behind a prefix": ((1, 2, 128, 16, "bf16", False), 8, [700 + 3 * i for i in range(24)], [1] * 24,
                             tuple((i, 0, 43) for i in range(1, 24)), "layer", (0, 0)),
    "many behind a prefix, fp8": ((2, 1, 96, 8, "fp8_e4m3", True), 8, [700 + 3 * i for i in range(17)], [1] * 17,
                                  tuple((i, 0, 80) for i in range(1, 17)), "layer", (0, 0)),
    "many behind a prefix, d 256": ((1, 1, 256, 8, "bf16", False), 8, [400 + 3 * i for i in range(17)], [1, 2] * 8 + [1],
                                    tuple((i, 0, 45) for i in range(1, 17)), "layer", (0, 0)),
}


@pytest.mark.parametrize("name", list(ATTN))
@pytest.mark.parametrize("with_weights", [False, True])
def test_attention(gpu, name, with_weights):
    import torch
    (L, H, D, B, dtype, scales), G, lens, q_lens, shared, layout, (pad, off) = ATTN[name]
    N = sum(-(-n // B) for n in lens) + 3
    g = W.Geometry(L, H, D, B, dtype, N, scales=scales)
    p = Pool(gpu, g, layout, seed=len(name))
    rows = _tables(p.rng, N, lens, B, shared)
    p.fill(rows, lens)
    for io_name in ([dtype] if dtype != "fp8_e4m3" else ["bf16", "f16"]):
        io = _torch_type(io_name)
        T, Hq, layer, scale = sum(q_lens), G * H, L - 1, 1.5 * D ** -0.5
        q = _heads(torch, gpu, p.rng.standard_normal((T, Hq, D)), io, pad, off)
        out = _heads(torch, gpu, np.zeros((T, Hq, D)), io, pad, off)
        lse = torch.full((T, Hq), 7.0, device=gpu)
        cap = max(lens) + 3
        before = p.rng.uniform(0, 2, (len(lens), H, cap)).astype(np.float32)
        weights = torch.from_numpy(before).to(gpu) if with_weights else None
        o, ids = R.csr(rows)
        kv.kv_check(p.batch.set(o, ids, lens, q_lens, Hq))
        kv.kv_check(p.batch.attn(layer, q, out, scale, lse=lse if not with_weights or io_name == "bf16" else None, weights=weights))
        torch.cuda.synchronize()
        ref, tol, rlse, ltol, rw, wtol = R.attention(p.values()[layer], rows, lens, q_lens, q.double().cpu().numpy(), scale, io_name, B)
        got = out.double().cpu().numpy()
        assert np.isfinite(got).all()
        assert (np.abs(got - ref) <= tol).all(), np.abs(got - ref).max()
        if not with_weights or io_name == "bf16":
            gl = lse.double().cpu().numpy()
            assert np.array_equal(np.isinf(gl), np.isinf(rlse))
            fin = np.isfinite(rlse)
            assert (np.abs(gl[fin] - rlse[fin]) <= ltol[fin]).all()
        if with_weights:
            w = weights.cpu().numpy().astype(np.float64)
            for i, n in enumerate(lens):
                want = before[i].astype(np.float64)
                want[:, :n] += rw[i]
                bound = np.full(want.shape, 0.0)
                bound[:, :n] = wtol[i] + 2.0 ** -22 * np.abs(want[:, :n]) + 1e-30
                assert (np.abs(w[i] - want) <= bound).all()
        # everything else around the outputs is untouched: the padding still holds NaN
        if pad:
            whole = out.as_strided((T, Hq, D + pad), (out.stride(0), out.stride(1), 1), out.storage_offset())
            assert torch.isnan(whole[..., D:].float()).all()


def test_attention_twice_gives_the_same_bits(gpu):
    import torch
    (L, H, D, B, dtype, scales), G, lens, q_lens, shared, _, _ = ATTN["many behind a prefix"]
    N = sum(-(-n // B) for n in lens) + 3
    p = Pool(gpu, W.Geometry(L, H, D, B, dtype, N), seed=3)
    rows = _tables(p.rng, N, lens, B, shared)
    p.fill(rows, lens)
    q = torch.randn(sum(q_lens), G * H, D, device=gpu).bfloat16()
    o, ids = R.csr(rows)
    kv.kv_check(p.batch.set(o, ids, lens, q_lens, G * H))
    got = []
    for _ in range(3):
        out, lse, w = torch.empty_like(q), torch.empty(q.shape[:2], device=gpu), torch.zeros(len(lens), H, max(lens), device=gpu)
        kv.kv_check(p.batch.attn(0, q, out, D ** -0.5, lse=lse, weights=w))
        got.append((out.view(torch.int16), lse.view(torch.int32), w.view(torch.int32)))
    for x in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(x, got[0]))


@pytest.mark.parametrize("what", ["nan", "inf"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8_e4m3"])
def test_rows_do_not_feel_tokens_that_they_do_not_see(gpu, dtype, what):
    """New token 70 of a prompt holds NaN or infinities: rows in front of it are as without them, rows from it on are not finite."""
    import torch
    if dtype == "fp8_e4m3" and what == "inf":
        pytest.skip("the type has no infinity")
    H, D, B, G, n, bad = 2, 128, 16, 4, 150, 70
    p = Pool(gpu, W.Geometry(1, H, D, B, dtype, 12), seed=5)
    rows = _tables(p.rng, 12, [n], B)
    p.fill(rows, [n])
    io_name = "f16" if dtype == "f16" else "bf16"
    q = torch.from_numpy(p.rng.standard_normal((n, G * H, D))).to(_torch_type(io_name)).to(gpu)
    ref, tol, rlse, ltol, _, _ = R.attention(p.values()[0], rows, [n], [n], q.double().cpu().numpy(), D ** -0.5, io_name, B)
    bits = {"fp8_e4m3": 0x7F, "bf16": 0x7FC0 if what == "nan" else 0x7F80, "f16": 0x7E00 if what == "nan" else 0x7C00}[dtype]
    p.bits()[0, :, int(rows[0][bad // B]), bad % B] = bits
    o, ids = R.csr(rows)
    out, lse = torch.empty_like(q), torch.empty(n, G * H, device=gpu)
    kv.kv_check(p.batch.set(o, ids, [n], [n], G * H))
    kv.kv_check(p.batch.attn(0, q, out, D ** -0.5, lse=lse))
    got = out.double().cpu().numpy()
    assert (np.abs(got[:bad] - ref[:bad]) <= tol[:bad]).all()
    assert (np.abs(lse.double().cpu().numpy()[:bad] - rlse[:bad]) <= ltol[:bad]).all()
    assert not np.isfinite(got[bad:]).any()


@pytest.mark.parametrize("shape", [(2, 72, 5, 3), (1, 64, 16, 8), (2, 192, 4, 2), (1, 256, 32, 4)])
@pytest.mark.parametrize("new", [2, 5, 90])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8_e4m3"])
def test_rows_do_not_feel_tokens_that_they_do_not_see_in_any_kernel(gpu, dtype, new, shape):
    """The same for few and many new tokens and other shapes, with several such tokens, one of them one that all rows see but the first."""
    import torch
    H, D, B, G = shape
    n = 170
    bad = sorted({n - 1, n - new + 1, n - new // 2})
    N = -(-n // B) + 2
    p = Pool(gpu, W.Geometry(1, H, D, B, dtype, N), seed=6)
    rows = _tables(p.rng, N, [n], B)
    p.fill(rows, [n])
    io_name = "f16" if dtype == "f16" else "bf16"
    q = torch.from_numpy(p.rng.standard_normal((new, G * H, D))).to(_torch_type(io_name)).to(gpu)
    ref, tol, _, _, _, _ = R.attention(p.values()[0], rows, [n], [new], q.double().cpu().numpy(), D ** -0.5, io_name, B)
    nan = {"fp8_e4m3": 0x7F, "bf16": 0x7FC0, "f16": 0x7E00}[dtype]
    for k, x in enumerate(bad):  # one element of V each, and all of K but for the first
        p.bits()[0, 1, int(rows[0][x // B]), x % B, :, 7 * k] = nan
        if k:
            p.bits()[0, 0, int(rows[0][x // B]), x % B] = nan
    o, ids = R.csr(rows)
    out = torch.empty_like(q)
    kv.kv_check(p.batch.set(o, ids, [n], [new], G * H))
    kv.kv_check(p.batch.attn(0, q, out, D ** -0.5))
    got = out.double().cpu().numpy()
    for j in range(new):
        seen = [k for k, x in enumerate(bad) if x <= n - new + j]
        if any(seen[1:]) or (seen and seen[0] > 0):
            assert np.isnan(got[j]).all(), j
        elif seen:
            assert np.isnan(got[j][:, 0]).all() and (np.abs(got[j] - ref[j]) <= tol[j])[:, 1:].all(), j
        else:
            assert (np.abs(got[j] - ref[j]) <= tol[j]).all(), j


@pytest.mark.parametrize("size", [1e-4, 2000.0])
@pytest.mark.parametrize("io_name", ["f16", "bf16"])
@pytest.mark.parametrize("B,q_lens", [(16, [1, 1]), (5, [1, 1]), (16, [60, 1]), (5, [60, 1])])
def test_scales_far_from_one(gpu, B, q_lens, io_name, size):
    """fp8 values with scales that weights times scale in f16 would not survive; blocks differ by a factor of up to eight."""
    import torch
    lens, H, G, D = [300, 70], 2, 4, 64
    N = sum(-(-n // B) for n in lens) + 3
    p = Pool(gpu, W.Geometry(1, H, D, B, "fp8_e4m3", N, scales=True), seed=11)
    rows = _tables(p.rng, N, lens, B)
    p.fill(rows, lens)
    small = torch.randn(2, N, B, H, D, generator=torch.Generator().manual_seed(1)).clamp_(-4, 4)
    used = ~torch.isnan(p.view[0].float())
    p.bits()[0] = torch.where(used, small.to(gpu).to(torch.float8_e4m3fn).view(torch.uint8), p.bits()[0])
    p.scale[0, 0].uniform_(0.5, 1.0)
    p.scale[0, 1].uniform_(size / 8, size)
    q = torch.from_numpy(p.rng.standard_normal((sum(q_lens), G * H, D))).to(_torch_type(io_name)).to(gpu)
    o, ids = R.csr(rows)
    out = torch.empty_like(q)
    kv.kv_check(p.batch.set(o, ids, lens, q_lens, G * H))
    kv.kv_check(p.batch.attn(0, q, out, D ** -0.5))
    ref, tol, _, _, _, _ = R.attention(p.values()[0], rows, lens, q_lens, q.double().cpu().numpy(), D ** -0.5, io_name, B)
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol + 2.0 ** -25).all()


def test_a_negative_scale_and_none(gpu):
    import torch
    for lens, q_lens in (([300, 70], [1, 1]), ([300, 70], [80, 1])):
        p = Pool(gpu, W.Geometry(1, 2, 128, 16, "bf16", 30), seed=8)
        rows = _tables(p.rng, 30, lens, 16)
        p.fill(rows, lens)
        o, ids = R.csr(rows)
        q = torch.from_numpy(p.rng.standard_normal((sum(q_lens), 8, 128))).bfloat16().to(gpu)
        kv.kv_check(p.batch.set(o, ids, lens, q_lens, 8))
        for scale in (-0.1, 0.0, -0.0):
            out, w = torch.empty_like(q), torch.zeros(2, 2, 300, device=gpu)
            kv.kv_check(p.batch.attn(0, q, out, scale, weights=w))
            ref, tol, _, _, rw, wtol = R.attention(p.values()[0], rows, lens, q_lens, q.double().cpu().numpy(), scale, "bf16", 16)
            assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()
            for i, n in enumerate(lens):
                assert (np.abs(w[i, :, :n].double().cpu().numpy() - rw[i]) <= wtol[i] + 2.0 ** -22 * rw[i]).all()


def test_attention_far_into_a_pool(gpu):
    """Blocks whose bytes lie beyond 4 GiB from the layer's first."""
    import torch
    g = W.Geometry(1, 8, 128, 16, "bf16", 150000)
    raw = torch.empty(g.pool_bytes, dtype=torch.uint8, device=gpu)
    arena = torch.empty(g.S, dtype=torch.uint8, device=gpu)
    kp = kv.KVPool(g, raw, arena, flags=kv.KV_STAGING_DEVICE)
    b = kv.KVBatch(kp)
    view = raw.view(torch.bfloat16).view(1, 2, g.N, g.B, g.H, g.D)
    rng = np.random.default_rng(0)
    rows = [np.array([149999, 3, 149998, 140000, 139999], np.int32), np.array([131072, 131071, 149000], np.int32)]
    lens, G = [77, 40], 4
    small = np.zeros((1, 2, 8, g.B, g.H, g.D))
    every = np.concatenate(rows)
    x = torch.randn(2, 8, g.B, g.H, g.D).bfloat16()
    view[0, :, torch.from_numpy(every).long().to(gpu)] = x.to(gpu)
    small[0] = x.double().numpy()
    q = torch.randn(2, G * 8, 128).bfloat16()
    out, lse = torch.empty_like(q, device=gpu), torch.empty(2, G * 8, device=gpu)
    o, ids = R.csr(rows)
    kv.kv_check(b.set(o, ids, lens, [1, 1], G * 8))
    kv.kv_check(b.attn(0, q.to(gpu), out, 128 ** -0.5, lse=lse))
    ref, tol, rlse, ltol, _, _ = R.attention(small[0], [np.arange(5), np.arange(5, 8)], lens, [1, 1], q.double().numpy(), 128 ** -0.5, "bf16", 16)
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()
    # and the way in: the last tokens again
    k, v = torch.randn(2, 8, 128).bfloat16(), torch.randn(2, 8, 128).bfloat16()
    kv.kv_check(b.append(0, None, k.to(gpu), v.to(gpu)))
    assert torch.equal(view[0, 0, 139999, 12].cpu(), k[0]) and torch.equal(view[0, 1, 149000, 7].cpu(), v[1])
    b.close()
    kp.close()


def test_calls_on_several_streams(gpu):
    """Set on one stream, used on two others, set again: the batch puts its calls behind each other."""
    import torch
    (L, H, D, B, dtype, scales), G, lens, q_lens, shared, _, _ = ATTN["long, few rows"]
    lens = [20011, 9]
    q_lens = [1, 1]
    N = sum(-(-n // B) for n in lens) + 3
    p = Pool(gpu, W.Geometry(L, H, D, B, dtype, N), seed=9)
    rows = _tables(p.rng, N, lens, B)
    p.fill(rows, lens)
    q = torch.randn(2, G * H, D, device=gpu).bfloat16()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    want = []
    for pick in ([0, 1], [1, 0]):
        out = torch.empty_like(q)
        o, ids = R.csr([rows[i] for i in pick])
        kv.kv_check(p.batch.set(o, ids, [lens[i] for i in pick], q_lens, G * H))
        kv.kv_check(p.batch.attn(0, q, out, D ** -0.5))
        torch.cuda.synchronize()
        want.append(out)
    for turn in range(6):
        outs = [torch.zeros_like(q) for _ in range(2)]
        torch.cuda.synchronize()
        for k, pick in enumerate(([0, 1], [1, 0])):
            o, ids = R.csr([rows[i] for i in pick])
            kv.kv_check(p.batch.set(o, ids, [lens[i] for i in pick], q_lens, G * H, stream=streams[(turn + k) % 3]))
            kv.kv_check(p.batch.attn(0, q, outs[k], D ** -0.5, stream=streams[(turn + k + 1) % 3]))
        torch.cuda.synchronize()
        for k in range(2):
            assert torch.equal(outs[k], want[k]), (turn, k)


def test_calls_in_a_graph(gpu):
    """Append, attention with weights and eviction captured once, replayed on new inputs."""
    import torch
    H, D, B, G, n = 2, 128, 16, 4, 300
    p = Pool(gpu, W.Geometry(2, H, D, B, "bf16", 50), seed=2)
    rows = _tables(p.rng, 50, [n, 70], B)
    p.fill(rows, [n, 70])
    o, ids = R.csr(rows)
    st = torch.cuda.Stream()
    q, k, v = (torch.randn(2, h, D, device=gpu).bfloat16() for h in (G * H, H, H))
    out, qo = torch.empty_like(q), torch.empty_like(q)
    w = torch.zeros(1, 2, H, n, device=gpu)
    w2, kept = torch.zeros_like(w), torch.full((1, 2, H, 64), -1, dtype=torch.int32, device=gpu)
    turns = torch.from_numpy(kv.kv_rope_freqs(D)[1]).to(gpu)
    start = p.bits().clone()

    def step():
        kv.kv_check(p.batch.append(1, q, k, v, qo, turns=turns, stream=st))
        kv.kv_check(p.batch.attn(1, qo, out, D ** -0.5, weights=w[0], stream=st))
        kv.kv_check(p.batch.evict(1, 1, w, kept, 64, 4, 8, weights_out=w2, stream=st))

    def again():
        p.bits().copy_(start)
        w.zero_()
        w2.zero_()
        torch.cuda.synchronize()

    torch.cuda.synchronize()
    kv.kv_check(p.batch.set(o, ids, [n, 70], [1, 1], G * H, stream=st))
    assert p.batch.set(o, ids, [n, 70], [1, 1], G * H, stream=st) == kv.KV_OK
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        assert p.batch.set(o, ids, [n, 70], [1, 1], G * H, stream=st) == kv.KV_EINVAL
        step()
    for turn in range(3):
        for x in (q, k, v):
            x.normal_()
        again()
        step()
        torch.cuda.synchronize()
        want = [x.clone() for x in (out, qo, w, w2, kept, p.bits())]
        for x in (out, qo, kept):
            x.zero_()
        again()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (out, qo, w, w2, kept, p.bits())):
            assert torch.equal(a.view(torch.uint8) if a.dtype.is_floating_point else a, b.view(torch.uint8) if b.dtype.is_floating_point else b), turn


APPEND = {
    # geometry, G (0: no queries), lens, q_lens, rot, interleaved, (pad, off), positions run ahead by
    "one token": ((1, 1, 64, 16, "bf16", False), 1, [1], [1], 64, False, (0, 0), 0),
    "decode": ((2, 4, 64, 16, "f16", False), 2, [5, 16, 17, 0, 300], [1, 1, 1, 1, 1], 64, True, (0, 0), 0),
    "prompts": ((1, 2, 128, 16, "bf16", False), 4, [200, 41], [200, 7], 128, False, (0, 0), 0),
    "far positions": ((1, 2, 128, 16, "f16", False), 2, [40, 41], [2, 7], 128, False, (0, 0), 2000000000),
    "part of the head": ((1, 2, 80, 5, "f16", False), 3, [90, 33], [4, 33], 54, False, (0, 0), 7),
    "part of the head, interleaved": ((1, 3, 72, 5, "bf16", False), 1, [90, 33], [4, 33], 30, True, (3, 5), 7),
    "two elements": ((1, 1, 128, 1, "bf16", False), 2, [9], [3], 2, False, (0, 0), 7),
    "nothing turned": ((1, 1, 128, 1, "bf16", False), 2, [9], [3], 0, False, (0, 0), 7),
    "no queries": ((1, 2, 112, 16, "f16", False), 0, [90, 33], [4, 33], 112, False, (1, 1), 0),
    "d 256": ((1, 2, 256, 16, "f16", False), 2, [90, 33], [4, 33], 256, False, (0, 0), 0),
    "d 256, interleaved": ((1, 2, 256, 16, "bf16", False), 2, [90, 33], [4, 33], 128, True, (8, 8), 0),
    "fp8": ((2, 2, 128, 32, "fp8_e4m3", False), 4, [50, 7], [9, 1], 128, False, (0, 0), 0),
    "fp8 with scales": ((2, 4, 128, 32, "fp8_e4m3", True), 2, [50, 70, 1], [40, 1, 1], 64, False, (0, 0), 0),
    "fp8 with scales, odd": ((2, 2, 72, 6, "fp8_e4m3", True), 2, [50, 70, 1], [40, 1, 1], 72, True, (0, 0), 100000),
    "fp8 with scales, strides of 2 bytes": ((2, 2, 96, 4, "fp8_e4m3", True), 2, [50, 70, 1], [40, 1, 1], 34, False, (1, 3), 0),
}


@pytest.mark.parametrize("name", list(APPEND))
@pytest.mark.parametrize("layout", ["layer", "block"])
def test_append(gpu, name, layout):
    import torch
    (L, H, D, B, dtype, scales), G, lens, q_lens, rot, inter, (pad, off), ahead = APPEND[name]
    N = sum(-(-n // B) for n in lens) + 3
    g = W.Geometry(L, H, D, B, dtype, N, scales=scales)
    p = Pool(gpu, g, layout, seed=len(name))
    rows = _tables(p.rng, N, lens, B)
    p.fill(rows, lens)
    layer = L - 1
    magnitude = 1.25
    freq = 500000.0 ** (-np.arange(rot // 2) * 2.0 / max(rot, 1)) / (2 * np.pi)
    words = np.array([int(round(f * 2.0 ** 64)) for f in freq], np.int64)
    turns = torch.from_numpy(words).to(gpu) if rot else None
    T = sum(q_lens)
    index = np.concatenate([np.arange(n - q, n) if n else np.array([-1]) for n, q in zip(lens, q_lens)])
    req = np.repeat(np.arange(len(lens)), q_lens)
    pos = index + ahead
    o, ids = R.csr(rows)
    for io_name in ([dtype] if dtype != "fp8_e4m3" else ["bf16", "f16"]):
        io, u = _torch_type(io_name), R.U[io_name]
        new = lambda n: _heads(torch, gpu, p.rng.standard_normal((T, n, D)) * (1.0 if dtype != "fp8_e4m3" else 20.0), io, pad, off)  # noqa: E731
        q = new(G * H) if G else None
        k, v = new(H), new(H)
        q_out = _heads(torch, gpu, np.zeros((T, max(G, 1) * H, D)), io, pad, off) if G else None
        scale = [torch.from_numpy(p.rng.uniform(0.03, 0.06, H).astype(np.float32)).to(gpu) for _ in range(2)] if scales else [None, None]
        before, sbefore = p.bits().clone(), None if p.scale is None else p.scale.clone()
        kv.kv_check(p.batch.set(o, ids, lens, q_lens, max(G, 1) * H))
        kv.kv_check(p.batch.append(layer, q, k, v, q_out, turns=turns, interleaved=inter, magnitude=magnitude,
                                   positions=torch.from_numpy(pos.astype(np.int32)).to(gpu) if ahead else None, k_scale=scale[0], v_scale=scale[1]))
        torch.cuda.synchronize()
        slop = 2.0 ** -15  # of the products' magnitudes: what cosines, sines and the products in 32 bits may be off by
        if G:
            ref, mag = R.rotate(q.double().cpu().numpy(), pos, freq, magnitude, inter)
            assert (np.abs(q_out.double().cpu().numpy() - ref) <= u * np.abs(ref) + 2 * slop * mag + 2.0 ** -25).all()
        rk, mk = R.rotate(k.double().cpu().numpy(), pos, freq, magnitude, inter)
        rv = v.double().cpu().numpy()
        live = index >= 0
        blk = np.array([rows[r][x // B] if x >= 0 else 0 for r, x in zip(req, index)])[live].astype(np.int64)
        place = (index % B)[live]
        stored = p.view.contiguous().cpu().float().numpy().astype(np.float64)[layer]
        for c, ref, mag in ((0, rk, mk), (1, rv, np.abs(rv) * 0)):
            ref, mag = ref[live], mag[live]
            got = stored[c, blk, place]
            if dtype == "fp8_e4m3":
                if scales:
                    s = scale[c].double().cpu().numpy()[None, :, None]
                    ref, mag = ref / s, mag / s
                ref = np.clip(ref, -448, 448)
                assert (np.abs(got - ref) <= 2.0 ** -4 * np.abs(ref) + 2.0 ** -10 + 2 * slop * mag).all()
            else:
                assert (np.abs(got - ref) <= u * np.abs(ref) + 2 * slop * mag + 2.0 ** -25).all()
        # nothing else of the pool has changed
        mask = torch.zeros(g.N, g.B, dtype=torch.bool, device=gpu)
        mask[torch.from_numpy(blk).to(gpu), torch.from_numpy(place).to(gpu)] = True
        same = p.bits() == before
        same[layer][:, mask] = True
        assert same.all()
        if scales:
            want = sbefore.clone()
            for c in range(2):
                want[layer, c, torch.from_numpy(blk).to(gpu)] = scale[c]
            assert torch.equal(want, p.scale)


def test_append_in_place_and_beyond_the_range(gpu):
    """q_out is q; an fp8 pool takes what is too large as its largest value, and a NaN as a NaN."""
    import torch
    g = W.Geometry(1, 2, 64, 16, "fp8_e4m3", 4)
    p = Pool(gpu, g)
    rows = [np.array([2], np.int32)]
    o, ids = R.csr(rows)
    kv.kv_check(p.batch.set(o, ids, [3], [1], 4))
    q = torch.randn(1, 4, 64, device=gpu).bfloat16()
    k = torch.randn(1, 2, 64, device=gpu).bfloat16()
    v = torch.tensor([1e30, -1e30, float("inf"), -float("inf"), 448.0, 449.0, float("nan"), 0.0] * 16, device=gpu).bfloat16().view(1, 2, 64)
    turns = torch.from_numpy(kv.kv_rope_freqs(64)[1]).to(gpu)
    apart, there = torch.empty_like(q), q.clone()
    kv.kv_check(p.batch.append(0, q, k, v, apart, turns=turns))
    kv.kv_check(p.batch.append(0, there, k, v, turns=turns))
    assert torch.equal(apart, there) and not torch.equal(there, q)
    got = p.view[0, 1, 2, 2].float().cpu().view(-1, 8)
    want = torch.tensor([448.0, -448.0, 448.0, -448.0, 448.0, 448.0, 0.0, 0.0])
    assert torch.isnan(got[:, 6]).all()
    got[:, 6] = 0
    assert (got == want).all()


EVICT = {
    # geometry, lens, keep, first, last, kind of weights
    "one head": ((1, 1, 64, 16, "bf16", False), [100], 30, 4, 8, "random"),
    "some stay": ((2, 2, 64, 16, "f16", False), [0, 1, 29, 30, 31, 200], 30, 4, 8, "random"),
    "keep nothing": ((1, 2, 64, 16, "f16", False), [40, 3], 0, 0, 0, "random"),
    "keep one": ((1, 2, 64, 16, "f16", False), [40, 3], 1, 0, 0, "random"),
    "first and last only": ((1, 2, 72, 5, "bf16", False), [90, 55], 20, 12, 8, "random"),
    "first only": ((1, 2, 80, 4, "bf16", False), [90, 55], 17, 17, 0, "random"),
    "last only": ((1, 2, 80, 4, "bf16", False), [90, 55], 17, 0, 17, "random"),
    "all alike": ((2, 3, 128, 16, "bf16", False), [500, 333], 100, 0, 0, "alike"),
    "ties": ((2, 3, 128, 16, "bf16", False), [700, 333], 200, 5, 30, "ties"),
    "an edge between two values": ((1, 2, 64, 16, "bf16", False), [400], 150, 20, 30, "edge"),
    "an edge at the lowest": ((1, 2, 64, 16, "bf16", False), [400], 150, 20, 30, "lowest"),
    "zeros of both signs": ((1, 2, 96, 1, "f16", False), [700, 333], 200, 5, 30, "zeros"),
    "special": ((1, 2, 96, 1, "f16", False), [700, 333], 200, 5, 30, "special"),
    "all but one": ((1, 2, 112, 8, "f16", False), [700, 700], 699, 5, 30, "random"),
    "long rows": ((2, 1, 64, 16, "bf16", False), [9000, 4097, 4096], 4000, 4, 100, "random"),
    "large blocks": ((1, 2, 64, 100, "bf16", False), [450, 150], 140, 3, 20, "random"),
    "d 256": ((1, 2, 256, 20, "bf16", False), [300, 150], 140, 3, 20, "random"),
    "fp8": ((2, 2, 128, 32, "fp8_e4m3", False), [300, 150], 64, 3, 20, "random"),
    "fp8 with scales": ((2, 2, 128, 32, "fp8_e4m3", True), [300, 150], 70, 3, 20, "random"),
    "fp8 with scales, odd": ((2, 2, 72, 6, "fp8_e4m3", True), [300, 150], 70, 13, 20, "random"),
    "fp8 with scales, token by token": ((2, 2, 64, 1, "fp8_e4m3", True), [300, 150], 70, 13, 20, "random"),
    "fp8 with scales, large blocks": ((2, 2, 64, 80, "fp8_e4m3", True), [300, 250], 170, 13, 20, "random"),
}


def _weights(rng, kind, shape):
    w = rng.uniform(0, 1, shape).astype(np.float32) ** 8
    if kind == "alike":
        w[:] = 0.5
    elif kind == "ties":
        w = np.round(w * 5).astype(np.float32) / 5
    elif kind == "zeros":
        w = np.where(rng.uniform(0, 1, shape) < 0.9, np.float32(0) * np.sign(rng.standard_normal(shape)), w).astype(np.float32)
    elif kind in ("edge", "lowest"):  # just as many as stay have one value, all others the one below it; the one value is the lowest that there is
        w[:] = np.nextafter(np.float32(0.5), np.float32(0)) if kind == "edge" else np.nan
        pick = rng.permutation(np.arange(20, 370))[:100]
        w[..., pick] = 0.5 if kind == "edge" else np.array(0xFF7FFFFF, np.uint32).view(np.float32)
    elif kind == "special":
        r = rng.uniform(0, 1, shape)
        w = np.where(r < 0.5, np.nan, np.where(r < 0.6, np.inf, np.where(r < 0.7, -np.inf, np.where(r < 0.8, -w, w * 1e-42)))).astype(np.float32)
    return w


@pytest.mark.parametrize("name", list(EVICT))
@pytest.mark.parametrize("in_place", [True, False])
def test_evict(gpu, name, in_place):
    import torch
    (L, H, D, B, dtype, scales), lens, keep, first, last, kind = EVICT[name]
    N = sum(-(-n // B) for n in lens) + 3
    g = W.Geometry(L, H, D, B, dtype, N, scales=scales)
    p = Pool(gpu, g, "block" if in_place else "layer", seed=len(name))
    rows = _tables(p.rng, N, lens, B)
    p.fill(rows, lens)
    layer, layers = (0, L) if in_place else (L - 1, 1)
    n, cap = len(lens), max(lens) + 2
    w0 = _weights(p.rng, kind, (layers, n, H, cap))
    w = torch.from_numpy(w0.copy()).to(gpu)
    w2 = w if in_place else torch.full_like(w, 9.0)
    kept = torch.full((layers, n, H, keep + 2), -5, dtype=torch.int32, device=gpu)
    before, stood, sbefore = p.bits().clone().cpu(), p.values(), None if p.scale is None else p.scale.cpu().numpy().astype(np.float64)
    o, ids = R.csr(rows)
    kv.kv_check(p.batch.set(o, ids, lens, [1 if x else 0 for x in lens], H))
    kv.kv_check(p.batch.evict(layer, layers, w, kept, keep, first, last, weights_out=None if in_place else w2))
    torch.cuda.synchronize()
    after, stands = p.bits().cpu(), p.values()
    snow = None if p.scale is None else p.scale.cpu().numpy().astype(np.float64)
    got_w, got_kept = w2.cpu().numpy(), kept.cpu().numpy()
    written = torch.zeros(L, g.N, g.B, dtype=torch.bool)
    for l in range(layers):
        for i, m in enumerate(lens):
            k = min(m, keep)
            table = np.asarray(rows[i], np.int64)
            x = np.arange(k)
            if m > keep:
                written[layer + l, torch.from_numpy(table[x // B]), torch.from_numpy(x % B)] = True
            for h in range(H):
                want = R.evict_kept(w0[l, i, h], m, keep, first, last)
                assert np.array_equal(got_kept[l, i, h, :k], want)
                assert (got_kept[l, i, h, k:] == -5).all()
                ww = np.concatenate([w0[l, i, h][want], np.zeros(m - k, np.float32)])
                assert np.array_equal(got_w[l, i, h, :m].view(np.uint32), ww.view(np.uint32))
                tail = w0[l, i, h, m:] if in_place else np.full(cap - m, 9.0, np.float32)
                assert np.array_equal(got_w[l, i, h, m:].view(np.uint32), tail.view(np.uint32))
                for c in range(2):
                    src = (layer + l, c, table[want // B], want % B, h)
                    dst = (layer + l, c, table[x // B], x % B, h)
                    if not scales:
                        assert np.array_equal(after.numpy()[dst], before.numpy()[src])
                        continue
                    if m <= keep:
                        continue
                    old = sbefore[layer + l, c, table[want // B], h]
                    for b in range(-(-k // B)):
                        part = slice(b * B, min(k, (b + 1) * B))
                        now = snow[layer + l, c, table[b], h]
                        assert now == (old[part].max() if part.stop > first // B * B else sbefore[layer + l, c, table[b], h])
                        a, z = stands[dst][part], stood[src][part]
                        assert (np.abs(a - z) <= np.where(old[part] == now, 0, 1)[:, None] * (2.0 ** -4 * np.abs(z) + 2.0 ** -10 * now) + 1e-6 * np.abs(z)).all()
    same = (after == before).all(-1)  # [L, 2, N, B, H]
    same[:, :] |= written[:, None, :, :, None]
    assert same.all()


EVICT_CHUNKS = {
    # as EVICT: rows enough for a wavefront each, and moves of many chunks
    "many rows": ((12, 32, 64, 16, "bf16", False), [200, 37, 1000], 30, 4, 8, "ties"),
    "many rows, special": ((12, 32, 64, 16, "f16", False), [200, 37, 1000], 170, 0, 1, "special"),
    "d 256": ((2, 2, 256, 4, "f16", False), [3000, 2900], 1500, 0, 0, "random"),
    "all but the first": ((2, 2, 128, 16, "bf16", False), [1000], 999, 0, 999, "random"),
    "fp8 with scales": ((1, 2, 256, 16, "fp8_e4m3", True), [900, 400], 350, 13, 20, "random"),
    "fp8 with scales, odd blocks": ((2, 2, 128, 20, "fp8_e4m3", True), [900, 400, 501], 500, 50, 0, "random"),
    "fp8 with scales, blocks larger than a chunk": ((1, 2, 256, 144, "fp8_e4m3", True), [900, 400], 350, 13, 20, "random"),
}


@pytest.mark.parametrize("name", list(EVICT_CHUNKS))
@pytest.mark.parametrize("in_place", [True, False])
def test_evict_in_chunks(gpu, name, in_place, monkeypatch):
    monkeypatch.setitem(EVICT, name, EVICT_CHUNKS[name])
    test_evict(gpu, name, in_place)


@pytest.mark.parametrize("dtype", ["bf16", "fp8_e4m3"])
def test_evict_first_in_a_graph(gpu, dtype):
    """A capture that finds no room for the order of the moves makes them one after the other."""
    import torch
    B, H, D, lens, keep = 16, 2, 256, [700, 333], 300
    p = Pool(gpu, W.Geometry(1, H, D, B, dtype, 70, scales=dtype == "fp8_e4m3"), seed=6)
    rows = _tables(p.rng, 70, lens, B)
    p.fill(rows, lens)
    o, ids = R.csr(rows)
    st = torch.cuda.Stream()
    w = torch.rand(1, 2, H, 700, device=gpu)
    w2, kept = torch.zeros_like(w), torch.zeros(1, 2, H, keep, dtype=torch.int32, device=gpu)
    start, scale = p.bits().clone(), None if p.scale is None else p.scale.clone()
    torch.cuda.synchronize()
    kv.kv_check(p.batch.set(o, ids, lens, [1, 1], H, stream=st))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        kv.kv_check(p.batch.evict(0, 1, w, kept, keep, 4, 8, weights_out=w2, stream=st))

    def result(run):
        p.bits().copy_(start)
        if scale is not None:
            p.scale.copy_(scale)
        w2.zero_()
        kept.zero_()
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        return [x.clone() for x in (p.bits(), w2, kept)] + ([] if scale is None else [p.scale.clone()])

    want = result(lambda: kv.kv_check(p.batch.evict(0, 1, w, kept, keep, 4, 8, weights_out=w2, stream=st)))
    assert not torch.equal(want[0], start)
    for turn in range(3):
        w.uniform_()
        want = result(lambda: kv.kv_check(p.batch.evict(0, 1, w, kept, keep, 4, 8, weights_out=w2, stream=st)))
        for a, b in zip(want, result(graph.replay)):
            assert torch.equal(a, b), turn


def test_evict_with_a_shared_prefix(gpu):
    """Requests that share blocks may be evicted as long as the shared ones stay whole."""
    import torch
    B, H, D = 16, 2, 64
    lens = [200, 150]
    p = Pool(gpu, W.Geometry(1, H, D, B, "bf16", 40), seed=4)
    rows = _tables(p.rng, 40, lens, B, ((1, 0, 3),))
    p.fill(rows, lens)
    o, ids = R.csr(rows)
    kv.kv_check(p.batch.set(o, ids, lens, [1, 1], H))
    w = torch.rand(1, 2, H, 200, device=gpu)
    kept = torch.zeros(1, 2, H, 90, dtype=torch.int32, device=gpu)
    before = p.bits().clone()
    assert p.batch.evict(0, 1, w, kept, 90, 47, 8) == kv.KV_EDUP  # block 2 of the three would be written
    assert torch.equal(p.bits(), before)
    kv.kv_check(p.batch.evict(0, 1, w, kept, 90, 48, 8))
    torch.cuda.synchronize()
    shared = torch.from_numpy(rows[0][:3]).long().to(gpu)
    assert torch.equal(p.bits()[:, :, shared], before[:, :, shared])
    assert not torch.equal(p.bits(), before)


def test_the_streaming_example(gpu):
    """Append, attention over a shared prefix, eviction and the swap in one loop: a request that was preempted and resumed into other blocks
    goes on as if it had not been.  Its prefix is no longer shared, so sums are taken in another order: 16-bit roundings apart."""
    from paper_2510_02758_amd import stream_demo
    kept, evicted, share = stream_demo.run()
    plain, again, _ = stream_demo.run(preempt_at=-1)
    assert evicted == again > 0 and share < 0.75
    assert kept.isfinite().all() and plain.isfinite().all()
    assert float((kept - plain).norm() / plain.norm()) < 0.05
