"""Where the attention's 16-bit arithmetic can go wrong, on a real MI355X: weights and scales far apart, and values that are not finite.
Against the definition in 64 bits."""
import numpy as np
import pytest

import ops_ref as R
from paper_2510_02758_amd import kvswap as kv
from paper_2510_02758_amd import workloads as W
from test_gpu_ops import Pool, _tables, _torch_type

pytestmark = pytest.mark.gpu


def _attend(p, rows, lens, q_lens, q, scale):
    import torch
    o, ids = R.csr(rows)
    out = torch.empty_like(q)
    kv.kv_check(p.batch.set(o, ids, lens, q_lens, q.shape[1]))
    kv.kv_check(p.batch.attn(0, q, out, scale))
    torch.cuda.synchronize()
    return out.double().cpu().numpy()


@pytest.mark.parametrize("drop", [8, 12, 14, 16, 18, 20])
@pytest.mark.parametrize("G", [4, 32])  # row tiles, big tiles
@pytest.mark.parametrize("B", [16, 5])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "fp8_e4m3"])
def test_many_small_weights_beside_a_large_one(gpu, dtype, B, G, drop):
    """One key that takes most of the weight and has no value, before many alike that lie `drop` below it: the output is what these have in
    all.  Scores are exact here; a weight is rounded once to 16 bits, and to no less than 2^-34 of the largest (f16), the output once."""
    import torch
    n, D = 20000, 64
    N = -(-n // B) + 2
    p = Pool(gpu, W.Geometry(1, 1, D, B, dtype, N), seed=1)
    rows = _tables(p.rng, N, [n], B)
    x = np.arange(n)
    at = (torch.from_numpy(rows[0].astype(np.int64)[x // B]).to(gpu), torch.from_numpy(x % B).to(gpu))
    values = torch.zeros(2, N, B, 1, D, device=gpu)
    values[0, at[0], at[1], 0, 0] = -float(drop)
    values[1, at[0], at[1]] = 1.0
    values[:, at[0][0], at[1][0]] = 0.0
    stored = values.to(_torch_type(dtype))
    p.bits()[0] = stored.view(torch.uint8 if dtype == "fp8_e4m3" else torch.int16)
    for io_name in ([dtype] if dtype != "fp8_e4m3" else ["bf16", "f16"]):
        q = torch.zeros(1, G, D, device=gpu, dtype=_torch_type(io_name))
        q[:, :, 0] = 1.0
        got = _attend(p, rows, [n], [1], q, 1.0)
        tail = (n - 1) * np.exp(-float(drop))
        want = tail / (1 + tail)
        u = R.U[io_name]
        tol = want * (2 * u + 2.0 ** -14) + ((n * 2.0 ** -34 + 2.0 ** -25) if io_name == "f16" else 0)
        assert (np.abs(got - want) <= tol).all(), (io_name, want, np.abs(got - want).max())


@pytest.mark.parametrize("io_name", ["f16", "bf16"])
@pytest.mark.parametrize("B", [16, 6])
@pytest.mark.parametrize("new,G", [(1, 4), (1, 32), (3, 4), (40, 4)])  # row tiles, big tiles; without and with tokens that some rows do not see
@pytest.mark.parametrize("D", [64, 72])
def test_value_scales_far_apart(gpu, D, new, G, B, io_name):
    """Blocks whose values have large scales, but which get little weight, or which a row does not see at all: neither takes the precision of the
    others away."""
    import torch
    n, light = 300, 200
    N = -(-n // B) + 2
    p = Pool(gpu, W.Geometry(1, 2, D, B, "fp8_e4m3", N, scales=True), seed=2)
    rows = _tables(p.rng, N, [n], B)
    p.fill(rows, [n])
    x = np.arange(n)
    blk, place = rows[0].astype(np.int64)[x // B], x % B
    values = torch.randn(2, N, B, 2, D, generator=torch.Generator().manual_seed(3)).clamp_(-4, 4)
    values[0] = 0.0
    light_at = (torch.from_numpy(blk[light:]), torch.from_numpy(place[light:]))
    values[0, light_at[0], light_at[1], :, 0] = -18.0  # a score of -18 beside 0
    used = torch.zeros(N, B, dtype=torch.bool)
    used[torch.from_numpy(blk), torch.from_numpy(place)] = True
    bits = values.to(torch.float8_e4m3fn).view(torch.uint8)
    bits[:, ~used] = 0x7F
    p.bits()[0] = bits.to(gpu)
    p.scale[0, 0] = 1.0
    p.scale[0, 1] = 1e-3
    # blocks of light tokens only that every row sees have large scales; the last block, which the last row alone sees whole, a huge one
    whole = [b for b in range(-(-light // B), (n - new) // B)]
    p.scale[0, 1, torch.from_numpy(rows[0].astype(np.int64)[whole]).to(gpu)] = 1e7
    last = (n - 1) // B
    first_row_of_last = max(0, last * B - (n - new))  # rows that see some of it
    if first_row_of_last:
        p.scale[0, 1, int(rows[0][last])] = 1e25
    q = torch.zeros(new, 2 * G, D, dtype=_torch_type(io_name), device=gpu)
    q[:, :, 0] = 1.0
    got = _attend(p, rows, [n], [new], q, 1.0)
    ref, tol, _, _, _, _ = R.attention(p.values()[0], rows, [n], [new], q.double().cpu().numpy(), 1.0, io_name, B)
    seen = first_row_of_last or new
    assert (np.abs(got - ref)[:seen] <= tol[:seen] + 2.0 ** -25).all(), (np.abs(got - ref) / tol)[:seen].max()


def _prefix_blocks(g, n):
    """Blocks of a prefix long enough for n requests with a row of more than 16 each to share it (kvswap.h), and no fewer than few share."""
    token = 2 * g.H * g.D * (1 if g.dtype == "fp8_e4m3" else 2)
    return -(-max(1024, -(-230000000 // (token * (n - 1)))) // g.B)


def _behind(rng, prefix, own):
    """Tables that begin with the same `prefix` blocks and go on with own[i] blocks of their own; the number of blocks."""
    perm, at, rows = rng.permutation(prefix + sum(own)).astype(np.int32), prefix, []
    for k in own:
        rows.append(np.concatenate([perm[:prefix], perm[at:at + k]]))
        at += k
    return rows


@pytest.mark.parametrize("n", [8, 17, 150])  # row tiles, one big tile, several
@pytest.mark.parametrize("B,D", [(16, 64), (16, 128), (16, 256), (6, 72)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8_e4m3"])
def test_rows_behind_a_prefix_are_as_precise_whatever_their_number(gpu, dtype, B, D, n):
    """Two tokens of a shared prefix with values 1 and -1 and scores 0 and -a, all others without weight: the output is tanh(a/2), a difference of
    weights.  These carry 16 bits and more (2^-16 of their sum), and the output is rounded once."""
    import torch
    H = 4
    shared = _prefix_blocks(W.Geometry(1, H, D, B, dtype, 1), max(n, 17))
    N, lens = shared + n, [shared * B + 1] * n
    p = Pool(gpu, W.Geometry(1, H, D, B, dtype, N), seed=4)
    rows = _behind(p.rng, shared, [1] * n)
    first = int(rows[0][0])
    values = torch.zeros(2, N, B, H, D, device=gpu)
    values[0, ..., 0] = -64.0
    values[0, first, 0, :, 0], values[0, first, 1, :, 0] = 0.0, -1.0
    values[1, first, 0], values[1, first, 1] = 1.0, -1.0
    p.bits()[0] = values.to(_torch_type(dtype)).view(torch.uint8 if dtype == "fp8_e4m3" else torch.int16)
    for io_name in ([dtype] if dtype != "fp8_e4m3" else ["bf16", "f16"]):
        q = torch.zeros(n, H, D)
        a = torch.linspace(0.3, 1.5, n).to(_torch_type(io_name))
        q[:, :, 0] = a.float()[:, None]
        q = q.to(gpu, _torch_type(io_name))
        got = _attend(p, rows, lens, [1] * n, q, 1.0)
        assert p.batch.query()["read_tokens"] == shared * B + n
        want = np.tanh(a.double().numpy() / 2)[:, None, None]
        tol = R.U[io_name] * want * (1 + 2.0 ** -7) + 2.0 ** -16
        assert (np.abs(got - want) <= tol).all(), (io_name, (np.abs(got - want) / tol).max())


ODD = {
    # H, D, B, G, lens, q_lens; lens 0: 40 tokens behind a prefix that all share
    "decode": (2, 128, 16, 4, [300, 70], [1, 1]),
    "decode, d 72": (2, 72, 6, 4, [300, 70], [1, 1]),
    "decode, d 256": (1, 256, 16, 4, [300, 70], [1, 1]),
    "decode, cut": (1, 64, 16, 4, [9000, 70], [1, 1]),
    "two new tokens": (2, 128, 16, 4, [300, 70], [2, 2]),
    "two new tokens, d 256": (1, 256, 16, 4, [300, 70], [2, 2]),
    "many heads": (1, 128, 16, 40, [300, 70], [1, 1]),
    "prompt": (2, 128, 16, 4, [300, 70], [180, 40]),
    "prompt, d 72": (2, 72, 6, 4, [300, 70], [180, 40]),
    "prompt, d 256": (1, 256, 16, 4, [300, 70], [180, 40]),
    "prefix, few": (2, 64, 16, 4, [0] * 4, [1] * 4),
    "prefix": (2, 64, 16, 4, [0] * 17, [1] * 17),
    "prefix, d 96": (2, 96, 5, 2, [0] * 17, [1] * 17),
}


@pytest.mark.parametrize("name", list(ODD))
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_infinities_among_the_values(gpu, dtype, name):
    """An infinity in a value makes that element of the rows that see it infinite, two of unlike sign or a NaN make it a NaN; other elements, and
    rows that do not see the token, are as without."""
    import torch
    H, D, B, G, lens, q_lens = ODD[name]
    rng = np.random.default_rng(7)
    if lens[0]:
        N = sum(-(-n // B) for n in lens) + 3
        rows = _tables(rng, N, lens, B)
    else:
        shared, own = _prefix_blocks(W.Geometry(1, H, D, B, dtype, 1), 17), -(-40 // B)
        rows, lens, N = _behind(rng, shared, [own] * len(lens)), [shared * B + 40] * len(lens), shared + own * len(lens)
    p = Pool(gpu, W.Geometry(1, H, D, B, dtype, N), seed=7)
    p.fill(rows, lens)
    q = torch.from_numpy(p.rng.standard_normal((sum(q_lens), H * G, D))).to(_torch_type(dtype)).to(gpu)
    clean, tol, _, _, _, _ = R.attention(p.values()[0], rows, lens, q_lens, q.double().cpu().numpy(), D ** -0.5, dtype, B)
    up, nan = {"bf16": (0x7F80, 0x7FC0), "f16": (0x7C00, 0x7E00)}[dtype]
    down = up - 0x8000  # (as a signed word)
    first, last, new = 5, lens[0] - 2, lens[0] - max(2, q_lens[0] // 2)
    #       token, element, bits; element 0: one infinity, 1: one below zero, 2: both, 3: twice the same, 4: NaN, 5 and 6: seen by later rows only
    odd = [(first, 0, up), (first, 1, down), (first, 2, up), (33, 2, down), (first, 3, up), (34, 3, up), (40, 4, nan), (last, 5, up), (last, 6, down),
           (new, 6, up), (new, D - 1, down)]
    for token, d, bits in odd:
        p.bits()[0, 1, int(rows[0][token // B]), token % B, :, d] = bits
    with np.errstate(invalid="ignore"):
        want, _, _, _, _, _ = R.attention(p.values()[0], rows, lens, q_lens, q.double().cpu().numpy(), D ** -0.5, dtype, B)
    got = _attend(p, rows, lens, q_lens, q, D ** -0.5)
    assert len(lens) == 2 or p.batch.query()["read_tokens"] < 2 * lens[0]
    assert np.isposinf(want).any() and np.isneginf(want).any() and np.isnan(want).any()
    assert np.array_equal(np.isposinf(got), np.isposinf(want))
    assert np.array_equal(np.isneginf(got), np.isneginf(want))
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = np.isfinite(want)
    assert (np.abs(got - clean)[fine] <= tol[fine]).all()
