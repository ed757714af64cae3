"""hm_quantize_* and hm_expert_matmul / _dw against 64-bit references."""
import numpy as np
import pytest
import torch

import layer_reference as R
from gpu_harness import dev
from paper_2508_09591_amd import binding as B

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
DTYPES = [torch.bfloat16, torch.float32]


def values(rng, *shape):
    """Values of many sizes: rows, blocks and single elements apart by powers of two, zeros among them."""
    x = rng.standard_normal(shape).astype(np.float32)
    x *= np.ldexp(1.0, rng.integers(-12, 12, shape[:-1] + (1,))).astype(np.float32)
    x *= np.ldexp(1.0, rng.integers(-6, 7, shape)).astype(np.float32)
    x[rng.random(shape) < 0.05] = 0.0
    return x


def strided(x, dtype, extra):
    """The matrix with rows `extra` elements further apart, off a vector's alignment where that is odd."""
    t = torch.full((x.shape[0] * (x.shape[1] + extra) + extra,), float("nan"), dtype=dtype, device="cuda")
    m = t[extra:].view(x.shape[0], x.shape[1] + extra)[:, :x.shape[1]]
    m.copy_(dev(x))
    return m


def poisoned(pair):
    for t in pair:
        t.view(torch.uint8).fill_(0xAB)
    return pair


def numbers(q):
    return q.float().cpu().numpy().astype(np.float64)


def codes(s):
    return s.cpu().numpy().astype(np.int64)


def offsets_of(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


# ---- 8 bits: every byte ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,C", [(1, 1), (1, 7168), (3, 127), (7, 128), (5, 129), (65, 511), (9, 512), (33, 513), (4, 1030), (130, 2056), (2, 4100)])
def test_rows(rows, C, dtype):
    rng = np.random.default_rng(rows + C)
    x = torch.from_numpy(values(rng, rows, C)).to(dtype).float().numpy()
    want, want_codes = R.rows8(x)
    for extra in (0, 8, 3):
        q, s = poisoned(B.alloc_rows8(rows, C))
        B.hm_quantize_rows(strided(x, dtype, extra), q, s)
        assert np.array_equal(numbers(q), want) and np.array_equal(codes(s), want_codes)
        assert not q.view(torch.uint8)[:, C:].any()


def edge_values():
    """A block for each: zeros, the least and the largest numbers, the border between two exponents, NaN and infinities."""
    x = np.zeros((12, 128), dtype=np.float32)
    x[1, 3] = 1e-45
    x[2] = 1.1754944e-38
    x[3, :2] = np.finfo(np.float32).max, -1.0
    x[4, :3] = 448.0, 1.0, -0.5
    x[5, :3] = np.nextafter(np.float32(448.0), np.float32(1e9)), 1.0, -0.5
    x[6] = np.linspace(-448, 448, 128)
    x[7, :4] = np.nan, 2.0, -3.0, 5.0
    x[8, :4] = np.inf, -np.inf, 1.0, 100.0
    x[9] = np.nan
    x[10, :6] = 1.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -12, -2.0 ** -11
    x[11, :9] = 448.0, 17.0, 19.0, 21.0, 23.0, 1.0625, 1.1875, 9.5, 8.5   # ties
    return x


def test_edges_of_the_number_range():
    x = edge_values()
    want, want_codes = R.rows8(x)
    q, s = poisoned(B.alloc_rows8(*x.shape))
    B.hm_quantize_rows(dev(x), q, s)
    assert np.array_equal(numbers(q), want, equal_nan=True) and np.array_equal(codes(s), want_codes)
    off = np.array([0, 128], dtype=np.int32)
    want, want_codes, there = R.columns8(x.T.copy(), off)
    q, s = poisoned(B.alloc_columns8(128, 1, 12))
    B.hm_quantize_columns(dev(x.T.copy()), dev(off), q, s)
    assert there.tolist() == [True, False]
    assert np.array_equal(numbers(q)[:, :128], want[:, :128], equal_nan=True) and np.array_equal(codes(s)[:1], want_codes[:1])
    w = np.zeros((12, 64, 70), dtype=np.float32)
    w[:, :8, 3:19] = x.reshape(12, 8, 16)
    want = R.weights8(w)
    got = poisoned(B.alloc_weights8(12, 64, 70)) + poisoned(B.alloc_weights8(12, 70, 64))
    B.hm_quantize_weights(dev(w), *got)
    for i, (a, b) in enumerate(zip(got, want)):
        assert np.array_equal(numbers(a) if i % 2 == 0 else codes(a), b, equal_nan=True), i


COUNTS = [[1], [128], [129], [0, 5, 0], [300, 0, 1, 127, 128, 2], [0, 0, 0], [64] * 70, [1] * 130, [1000, 24], [0, 0, 256, 0]]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", [1, 64, 70, 200, 1030])
@pytest.mark.parametrize("counts", COUNTS)
def test_columns(counts, C, dtype):
    rng = np.random.default_rng(C + len(counts))
    off = offsets_of(counts)
    rows, spare = int(off[-1]), 3   # rows behind the last segment belong to none
    x = torch.from_numpy(values(rng, rows + spare, C)).to(dtype).float().numpy()
    want, want_codes, there = R.columns8(x, off)
    for extra in (0, 5):
        q, s = poisoned(B.alloc_columns8(rows + spare, len(counts), C))
        B.hm_quantize_columns(strided(x, dtype, extra), dev(off), q, s)
        got, got_codes = numbers(q).reshape(C, -1, 128), codes(s)
        assert np.array_equal(got[:, there], want.reshape(C, -1, 128)[:, there]) and np.array_equal(got_codes[there], want_codes[there])
        assert (q.view(torch.uint8).view(C, -1, 128)[:, dev(~there)] == 0xAB).all() and np.all(got_codes[~there] == 0xAB)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("E,N,C", [(1, 1, 1), (2, 128, 128), (3, 130, 7), (1, 7, 600), (5, 256, 512), (2, 1000, 300), (1, 640, 129)])
def test_weights(E, N, C, dtype):
    w = torch.from_numpy(values(np.random.default_rng(N + C), E, N, C)).to(dtype)
    want = R.weights8(w.float().numpy())
    got = poisoned(B.alloc_weights8(E, N, C)) + poisoned(B.alloc_weights8(E, C, N))
    B.hm_quantize_weights(w.cuda(), *got)
    for i, (a, b) in enumerate(zip(got, want)):
        assert np.array_equal(numbers(a) if i % 2 == 0 else codes(a), b), i
    alone = poisoned(B.alloc_weights8(E, N, C))
    B.hm_quantize_weights(w.cuda(), *alone)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(alone, got[:2]))


# ---- products -------------------------------------------------------------------------------------------------------
def operand(rng, *shape):
    """Random bytes that are numbers, with zeros, and random codes around 127."""
    q = rng.integers(0, 256, shape, dtype=np.uint8)
    q[(q & 0x7F) == 0x7F] = 0
    return q


def f8(bits):
    return torch.from_numpy(bits).view(F8)


def bound(want, size, largest, count, dtype):
    """bf16: the result is rounded (2^-9), and of a step's 64 products each may lose 2^-13 of the largest; twice 64 a block.
    fp32: each of the additions rounds by 2^-24 of what it adds to, here of the sum of magnitudes."""
    if dtype == torch.bfloat16:
        return 2.0 ** -8 * np.abs(want) + 128 * 2.0 ** -13 * largest + 1e-37
    return (count + 8) * 2.0 ** -24 * size + 1e-37


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,H", [(1, 1), (16, 128), (33, 129), (130, 512), (64, 1030), (257, 300), (1000, 640), (4, 2056)])
@pytest.mark.parametrize("counts", [[1], [0, 5, 0, 1], [130, 0, 1, 127, 128, 2], [3] * 70, [0, 0], [513], [16, 17, 31, 32, 33, 64, 65]])
def test_products_of_rows(counts, N, H, dtype):
    rng = np.random.default_rng(N * H + len(counts))
    off, E, spare = offsets_of(counts), len(counts), 2
    rows = int(off[-1]) + spare
    W = R.up(H, 128)
    x, w = operand(rng, rows, W), operand(rng, E, N, W)
    x[:, H:], w[:, :, H:] = 0, 0
    xs = rng.integers(120, 135, (rows, R.up(H, 512) // 128), dtype=np.uint8)
    ws = rng.integers(115, 130, (E, R.up(N, 128) // 128, R.up(H, 512) // 128), dtype=np.uint8)
    out = torch.full((rows, N), -77.0, dtype=dtype, device="cuda")
    B.hm_expert_matmul(f8(x).cuda(), dev(xs), f8(w).cuda(), dev(ws), dev(off), out)
    a = R.row_values(f8(x).float().numpy().astype(np.float64), xs.astype(np.int64))
    b = R.weight_values(f8(w).float().numpy().astype(np.float64), ws.astype(np.int64))
    got = out.float().cpu().numpy().astype(np.float64)
    assert np.all(got[off[-1]:] == -77.0)
    for e in range(E):
        r = slice(off[e], off[e + 1])
        if counts[e] == 0:
            continue
        want, size, largest = R.product(a[r], b[e], W // 128)
        assert np.all(np.abs(got[r] - want) <= bound(want, size, largest, W, dtype)), (e, np.abs(got[r] - want).max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,H", [(1, 1), (16, 128), (33, 129), (130, 70), (257, 300)])
@pytest.mark.parametrize("counts", [[1], [0, 5, 0, 1], [130, 0, 1, 127, 128, 2], [3] * 70, [0, 0], [700]])
def test_products_of_columns(counts, N, H, dtype):
    rng = np.random.default_rng(N * H + len(counts))
    off, E = offsets_of(counts), len(counts)
    rows = int(off[-1])
    blocks = rows // 128 + E
    gy, x = operand(rng, N, 128 * blocks), operand(rng, H, 128 * blocks)
    there = np.zeros(128 * blocks, dtype=bool)
    for e in range(E):
        first = 128 * (off[e] // 128 + e)
        there[first:first + counts[e]] = True
        for q in (gy, x):   # zeros behind a segment up to a whole block; what is in no segment's block may be anything
            q[:, first + counts[e]:first + R.up(counts[e], 128)] = 0
    gs, xs = rng.integers(120, 135, (blocks, N), dtype=np.uint8), rng.integers(115, 130, (blocks, H), dtype=np.uint8)
    dw = torch.full((E, N, H), -77.0, dtype=dtype, device="cuda")
    B.hm_expert_matmul_dw(f8(gy).cuda(), dev(gs), f8(x).cuda(), dev(xs), dev(off), rows, dw)
    a = R.column_values(f8(gy).float().numpy().astype(np.float64), gs.astype(np.int64))
    b = R.column_values(f8(x).float().numpy().astype(np.float64), xs.astype(np.int64))
    got = dw.float().cpu().numpy().astype(np.float64)
    for e in range(E):
        first, n = 128 * (off[e] // 128 + e), R.up(counts[e], 128)
        want, size, largest = R.product(a[first:first + n].T, b[first:first + n].T, n // 128)
        assert np.all(np.abs(got[e] - want) <= bound(want, size, largest, n, dtype)), (e, np.abs(got[e] - want).max())


def test_a_nan_stays_in_its_row_and_column():
    """NaN codes, in values and in scales, reach the results they are part of and no others."""
    rows, N, H, E = 40, 48, 256, 2
    rng = np.random.default_rng(1)
    x, w = operand(rng, rows, H), operand(rng, E, N, H)
    xs, ws = np.full((rows, 4), 127, dtype=np.uint8), np.full((E, 1, 4), 127, dtype=np.uint8)
    x[3, 200], w[1, 5, 0], xs[7, 1] = 0x7F, 0xFF, 255
    off = np.array([0, 20, 40], dtype=np.int32)
    for dtype in DTYPES:
        out = torch.zeros((rows, N), dtype=dtype, device="cuda")
        B.hm_expert_matmul(f8(x).cuda(), dev(xs), f8(w).cuda(), dev(ws), dev(off), out)
        bad = torch.isnan(out).cpu().numpy()
        want = np.zeros((rows, N), dtype=bool)
        want[3], want[20:, 5], want[7] = True, True, True
        assert np.array_equal(bad, want)


@pytest.mark.parametrize("rows,E,N,H", [(1, 1, 40, 128), (3, 1, 17, 129), (8, 32, 64, 640), (16, 1, 33, 2056), (24, 8, 100, 300)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_few_rows_are_summed_in_32_bits(rows, E, N, H, dtype):
    """Whole numbers beside products of 448 x 448 that cancel: every partial sum lies below 2^24 and the results below 2^8, so
    that sums in 32 bits, in any order, and their rounding to bf16 are exact."""
    rng = np.random.default_rng(rows + N + H)
    x, w = rng.integers(-2, 3, (rows, H)).astype(np.float32), rng.integers(-2, 3, (E, N, H)).astype(np.float32)
    x[:, 64:], w[:, :, 64:] = 0, 0   # at most 64 products of at most 4
    for first in range(0, H - 1, 128):   # two that cancel in each block
        a, b = first + rng.permutation(min(128, H - first))[:2]
        x[:, a], x[:, b] = 448, -448
        w[:, :, a], w[:, :, b] = 448, 448
    off = offsets_of(np.bincount(rng.permutation(np.arange(rows) % E), minlength=E))
    W = R.up(H, 128)
    pad = lambda t: torch.nn.functional.pad(torch.from_numpy(t), (0, W - H)).to(F8).cuda()
    xs = torch.full((rows, R.up(H, 512) // 128), 127, dtype=torch.uint8, device="cuda")
    ws = torch.full((E, R.up(N, 128) // 128, R.up(H, 512) // 128), 127, dtype=torch.uint8, device="cuda")
    out = torch.full((rows, N), -77.0, dtype=dtype, device="cuda")
    B.hm_expert_matmul(pad(x), xs, pad(w), ws, dev(off), out)
    expert = np.repeat(np.arange(E), np.diff(off))
    want = np.einsum("rh,rnh->rn", x.astype(np.float64), w.astype(np.float64)[expert])
    assert np.abs(want).max() <= 256 and np.array_equal(out.double().cpu().numpy(), want)


def cancelling(rng, rows, H):
    """Whole numbers up to 2 in the first 64 columns, and 448 and -448 somewhere in every block, the same places in each row."""
    x = rng.integers(-2, 3, (rows, H)).astype(np.float32)
    x[:, 64:] = 0
    for first in range(0, H - 1, 128):
        a, b = first + rng.permutation(min(128, H - first))[:2]
        x[:, a], x[:, b] = 448, -448
    return x


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,E,N,H", [(40, 1, 33, 129), (300, 3, 130, 640), (2000, 5, 1500, 384), (8300, 8, 1000, 256)])
def test_full_sums_of_rows(rows, E, N, H, dtype):
    """Products that cancel, by tiles of each size, as in test_few_rows_are_summed_in_32_bits: exact in whatever order."""
    rng = np.random.default_rng(rows)
    x, w = cancelling(rng, rows, H), rng.integers(-2, 3, (E, N, H)).astype(np.float32)
    w[:, :, np.abs(x[0]) == 448] = 448
    off = offsets_of(np.bincount(rng.permutation(np.arange(rows) % E), minlength=E))
    W = R.up(H, 128)
    pad = lambda t: torch.nn.functional.pad(torch.from_numpy(t), (0, W - H)).to(F8).cuda()
    xs = torch.full((rows, R.up(H, 512) // 128), 127, dtype=torch.uint8, device="cuda")
    ws = torch.full((E, R.up(N, 128) // 128, R.up(H, 512) // 128), 127, dtype=torch.uint8, device="cuda")
    x8, w8, out = pad(x), pad(w), torch.full((rows, N), -77.0, dtype=dtype, device="cuda")
    want = [x[off[e]:off[e + 1]].astype(np.float64) @ w[e].astype(np.float64).T for e in range(E)]
    for stream in (None, torch.cuda.current_stream()):   # by either way into the library
        out.fill_(-77)
        B.hm_expert_matmul(x8, xs, w8, ws, dev(off), out, stream=stream, full_sums=True)
        assert np.array_equal(out.double().cpu().numpy(), np.concatenate(want))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("counts,N,H", [([40], 33, 129), ([130, 0, 257], 400, 300), ([300, 100, 128], 1500, 1541), ([200, 500], 4100, 3900)])
def test_full_sums_of_columns(counts, N, H, dtype):
    rng = np.random.default_rng(N)
    off, E = offsets_of(counts), len(counts)
    rows = int(off[-1])
    blocks = rows // 128 + E
    gy, x = np.zeros((N, 128 * blocks), dtype=np.float32), np.zeros((H, 128 * blocks), dtype=np.float32)
    for e in range(E):
        if counts[e]:
            first = 128 * (off[e] // 128 + e)
            part = slice(first, first + counts[e])
            gy[:, part], x[:, part] = cancelling(rng, N, counts[e]), rng.integers(-2, 3, (H, counts[e]))
            x[:, part][:, np.abs(gy[0, part]) == 448] = 448
    one = lambda n: torch.full((blocks, n), 127, dtype=torch.uint8, device="cuda")
    gy8, x8, dw = torch.from_numpy(gy).to(F8).cuda(), torch.from_numpy(x).to(F8).cuda(), torch.empty((E, N, H), dtype=dtype, device="cuda")
    for stream in (None, torch.cuda.current_stream()):
        dw.fill_(-77)
        B.hm_expert_matmul_dw(gy8, one(N), x8, one(H), dev(off), rows, dw, stream=stream, full_sums=True)
        for e in range(E):
            part = slice(128 * (off[e] // 128 + e), 128 * (off[e] // 128 + e) + R.up(counts[e], 128))
            want = torch.from_numpy(gy[:, part]).cuda().double() @ torch.from_numpy(x[:, part]).cuda().double().t().contiguous()
            assert torch.equal(dw[e].double(), want), e


def test_what_the_units_products_drop():
    """bf16 results of tiles where 8 columns are 1,000 times as large as the others.  Each of the 64 products of a step loses
    less than 2^-13 of the step's largest, either way alike: sqrt(64 / 3) 2^-13 = 2^-10.8 of it, and steps add as their squares; rounding,
    evenly within 2^-8 of a result's power of two, adds 2^-9.2 of their norm.  Taken over a matrix, where such sums are sharp."""
    rows, N, H = 2048, 512, 2048
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x, w = torch.randn((rows, H), generator=g, device="cuda"), torch.randn((1, N, H), generator=g, device="cuda") / H ** 0.5
    x[:, ::256] *= 1000
    off = dev(np.array([0, rows], dtype=np.int32))
    x8, w8 = B.hm_quantize_rows(x, *B.alloc_rows8(rows, H)), B.hm_quantize_weights(w, *B.alloc_weights8(1, N, H))
    out = torch.empty((rows, N), dtype=torch.bfloat16, device="cuda")
    B.hm_expert_matmul(*x8, *w8, off, out)
    a, b = gpu_values(x8[0], x8[1]), gpu_values(w8[0][0], w8[1][0].repeat_interleave(128, dim=0))
    want = a @ b.t().contiguous()
    most = lambda t: t.abs().view(t.shape[0], -1, 128).amax(dim=2).square()   # bounds the products of both steps of a block
    loss = 2.0 ** -10.8 * (2 * (most(a) @ most(b).t().contiguous()).sum()).sqrt()
    assert (out.double() - want).norm() <= ((2.0 ** -9 * want.norm()) ** 2 + loss ** 2).sqrt()


@pytest.mark.parametrize("low", [0, 1, 2, 3, 5])
@pytest.mark.parametrize("rows", [8, 300])
@pytest.mark.parametrize("dtype", DTYPES)
def test_the_least_scales(low, rows, dtype):
    """Codes from 0 on; fp32 results round values to multiples of 2^-133, which only codes below 3 have need of."""
    N, H = 64, 256
    rng = np.random.default_rng(rows + low)
    x, w = operand(rng, rows, H), operand(rng, 1, N, H)
    xs, ws = np.full((rows, 4), low, dtype=np.uint8), np.full((1, 1, 4), 240, dtype=np.uint8)
    out = torch.zeros((rows, N), dtype=dtype, device="cuda")
    B.hm_expert_matmul(f8(x).cuda(), dev(xs), f8(w).cuda(), dev(ws), dev(np.array([0, rows], dtype=np.int32)), out)
    a = R.row_values(f8(x).float().numpy().astype(np.float64), xs.astype(np.int64))
    b = R.weight_values(f8(w).float().numpy().astype(np.float64), ws.astype(np.int64))[0]
    want, size, largest = R.product(a, b, H // 128)
    lost = 2.0 ** -133 * np.abs(b).sum(axis=1)[None, :] if dtype == torch.float32 and low < 3 else 0.0
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= bound(want, size, largest, H, dtype) + lost)


@pytest.mark.parametrize("full", [False, True])
@pytest.mark.parametrize("rows", [8, 300])
@pytest.mark.parametrize("dtype", DTYPES)
def test_the_largest_scales(rows, dtype, full):
    """Codes 246 with any value and 247 with values up to 240 hold numbers below 2^128 and lose nothing; from 2^128 on values of sums in
    32 bits are infinite, which the numbers next to fp32's and bf16's largest are rounded to."""
    N, H = 64, 256
    rng = np.random.default_rng(rows)
    x, w = operand(rng, rows, H), operand(rng, 1, N, H)
    x[:, 128:] = np.where((x[:, 128:] & 0x7F) > 0x77, 0, x[:, 128:])   # 0x77: 240
    xs, ws = np.full((rows, 4), 246, dtype=np.uint8), np.full((1, 1, 4), 20, dtype=np.uint8)
    xs[:, 1] = 247
    off = dev(np.array([0, rows], dtype=np.int32))
    out = torch.zeros((rows, N), dtype=dtype, device="cuda")
    B.hm_expert_matmul(f8(x).cuda(), dev(xs), f8(w).cuda(), dev(ws), off, out, full_sums=full)
    a = R.row_values(f8(x).float().numpy().astype(np.float64), xs.astype(np.int64))
    b = R.weight_values(f8(w).float().numpy().astype(np.float64), ws.astype(np.int64))[0]
    want, size, largest = R.product(a, b, H // 128)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= bound(want, size, largest, H, dtype))
    lowest = np.full((rows, H), np.finfo(np.float32).min, dtype=np.float32)
    x8 = B.hm_quantize_rows(dev(lowest), *B.alloc_rows8(rows, H))
    assert (x8[1][:, :2] == 247).all() and (x8[0].float() == -256).all()
    w8 = B.hm_quantize_weights(torch.full((1, N, H), 2.0 ** -20, device="cuda"), *B.alloc_weights8(1, N, H))
    B.hm_expert_matmul(*x8, *w8, off, out, full_sums=full)
    if dtype == torch.float32 or full or rows <= 16:
        assert (out == float("-inf")).all()
    else:
        assert (out == -2.0 ** (128 - 20 + 8)).all()


def test_offsets_that_are_wrong_stay_inside():
    """Descending offsets and offsets outside the rows: nothing outside the outputs is written."""
    rows, N, H = 50, 40, 128
    rng = np.random.default_rng(2)
    for off in ([-5, 20, 70], [40, 10, 50], [2 ** 31 - 1, -2 ** 31, 30], [0, 50, 0]):
        off = np.array(off, dtype=np.int32)
        x, xs = B.alloc_rows8(rows, H)
        w, ws = B.alloc_weights8(2, N, H)
        for t in (x, xs, w, ws):
            t.view(torch.uint8).fill_(56)
        guard = torch.full((rows + 2, N), 5.0, device="cuda")
        B.hm_expert_matmul(x, xs, w, ws, dev(off), guard[1:rows + 1])
        assert (guard[0] == 5).all() and (guard[-1] == 5).all()
        blocks = rows // 128 + 2
        room = torch.full((N * 128 * blocks + 512,), 7, dtype=torch.uint8, device="cuda")
        scale = torch.full((blocks * N + 64,), 7, dtype=torch.uint8, device="cuda")
        B.hm_quantize_columns(torch.ones((rows, N), device="cuda"), dev(off), room[256:-256].view(N, 128 * blocks), scale[32:-32].view(blocks, N))
        assert (room[:256] == 7).all() and (room[-256:] == 7).all() and (scale[:32] == 7).all() and (scale[-32:] == 7).all()
        xt, xts = B.alloc_columns8(rows, 2, N)
        for t in (xt, xts):
            t.view(torch.uint8).fill_(56)
        guard = torch.full((4, N, N), 5.0, device="cuda")
        B.hm_expert_matmul_dw(xt, xts, xt, xts, dev(off), rows, guard[1:3])
        assert (guard[0] == 5).all() and (guard[-1] == 5).all()


def test_nothing_to_do():
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    out = torch.empty((0, 40), device="cuda")
    B.hm_expert_matmul(*B.alloc_rows8(0, 128), *B.alloc_weights8(2, 40, 128), off, out)
    dw = torch.full((2, 40, 24), 3.0, device="cuda")
    B.hm_expert_matmul_dw(*B.alloc_columns8(0, 2, 40), *B.alloc_columns8(0, 2, 24), off, 0, dw)
    assert not dw.any()
    x = torch.empty((0, 40), device="cuda")
    B.hm_quantize_rows(x, *B.alloc_rows8(0, 40))
    B.hm_quantize_columns(x, off, *B.alloc_columns8(0, 2, 40))


@pytest.mark.parametrize("rows,E,N,H", [(4096, 4, 512, 1024), (300, 8, 384, 2048), (40, 16, 1024, 512), (3000, 3, 250, 640)])
def test_a_layer_of_products_and_their_gradients(rows, E, N, H):
    """y = x w, dx = gy w and dw = gy^T x of the values that the quantised operands stand for; on a stream of the caller's."""
    rng = np.random.default_rng(rows)
    off = np.sort(rng.integers(0, rows + 1, E - 1))
    off = np.concatenate([[0], off, [rows]]).astype(np.int32)
    x, w, gy = (torch.from_numpy(rng.standard_normal(s, dtype=np.float32)).cuda() for s in ((rows, H), (E, N, H), (rows, N)))
    d_off, stream = dev(off), torch.cuda.Stream()
    q = {k: poisoned(v) for k, v in {"x": B.alloc_rows8(rows, H), "gy": B.alloc_rows8(rows, N), "xt": B.alloc_columns8(rows, E, H),
                                     "gyt": B.alloc_columns8(rows, E, N), "w": B.alloc_weights8(E, N, H), "wt": B.alloc_weights8(E, H, N)}.items()}
    y, dx, dw = torch.empty((rows, N), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, H), device="cuda"), torch.empty((E, N, H), device="cuda")
    torch.cuda.synchronize()
    B.hm_quantize_rows(x, *q["x"], stream=stream)
    B.hm_quantize_rows(gy, *q["gy"], stream=stream)
    B.hm_quantize_columns(x, d_off, *q["xt"], stream=stream)
    B.hm_quantize_columns(gy, d_off, *q["gyt"], stream=stream)
    B.hm_quantize_weights(w, *q["w"], *q["wt"], stream=stream)
    B.hm_expert_matmul(*q["x"], *q["w"], d_off, y, stream=stream)
    B.hm_expert_matmul(*q["gy"], *q["wt"], d_off, dx, stream=stream)
    B.hm_expert_matmul_dw(*q["gyt"], *q["xt"], d_off, rows, dw, stream=stream)
    stream.synchronize()
    vx, vg = R.row_values(numbers(q["x"][0]), codes(q["x"][1]))[:, :H], R.row_values(numbers(q["gy"][0]), codes(q["gy"][1]))[:, :N]
    vw = R.weight_values(numbers(q["w"][0]), codes(q["w"][1]))[:, :, :H]
    near = lambda a, b, tol: np.linalg.norm(a - b) <= tol * np.linalg.norm(b)
    cols = [R.column_values(numbers(q[k][0]), codes(q[k][1])) for k in ("gyt", "xt")]
    for e in range(E):
        r = slice(off[e], off[e + 1])
        if off[e] == off[e + 1]:
            assert not dw[e].any()
            continue
        # rounding to bf16 is at most 2^-9 of each result; sums in 32 bits: sqrt(terms) 2^-24, with room
        assert near(y[r].double().cpu().numpy(), vx[r] @ vw[e].T, 2.0 ** -9 + 5e-5)
        assert near(dx[r].double().cpu().numpy(), vg[r] @ vw[e], 1e-5)
        first = 128 * (off[e] // 128 + e)
        a, b = (c[first:first + off[e + 1] - off[e]] for c in cols)
        assert near(dw[e].double().cpu().numpy(), a.T @ b, 1e-5)
        # the 8 bits themselves: e4m3 is good to 2^-4 of a value, and a sum of such errors averages out
        assert near(dw[e].double().cpu().numpy(), gy[r].double().cpu().numpy().T @ x[r].double().cpu().numpy(), 0.1)


def gpu_values(q, power):
    """[rows, k] values in 64 bits of operands [rows, k] and codes [rows, blocks]."""
    p = torch.ldexp(torch.ones((), dtype=torch.float64), power.cpu().int() - 127).cuda()   # exact on the host
    return (q.double().view(q.shape[0], -1, 128) * p[:, :, None]).view(q.shape[0], -1)


def same_in_every_patch(got, a, b, dtype):
    """The 2-norm of the error of a b^T in each 32 x 32 patch.  bf16: rounding is at most 2^-9 of a value, and of the 64 products
    of a step each may lose 2^-13 of the largest, which is no more than the largest of either block's values multiplied: twice
    64 * 2^-13 of that a block.  fp32: sums of some thousand terms in 32 bits, below 1e-5 of the patch."""
    want = a @ b.t().contiguous()
    R, C = got.shape
    cut = lambda t: torch.nn.functional.pad(t.double(), (0, -C % 32, 0, -R % 32)).view(-(-R // 32), 32, -(-C // 32), 32).square().sum(dim=(1, 3)).sqrt()
    most = lambda t: t.abs().view(t.shape[0], -1, 128).amax(dim=2)
    off, size = cut(got.double() - want), cut(want)
    bound = 2.0 ** -9 * size + 2.0 ** -6 * cut(most(a) @ most(b).t().contiguous()) if dtype == torch.bfloat16 else 1e-5 * size
    assert (off <= bound + 1e-30).all(), float((off / (bound + 1e-30)).max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H", [1, 129, 384, 512, 600, 1024, 1400])
@pytest.mark.parametrize("rows,E,N", [(2000, 5, 1500), (8300, 8, 2900), (2100, 1, 1541)])
def test_many_rows(rows, E, N, H, dtype):
    """Sizes whose tiles are large, with as many steps as end inside, at and behind a group of four; odd N cannot be stored in vectors."""
    rng = np.random.default_rng(rows + H)
    cuts = np.sort(rng.integers(0, rows - 3, E - 1)) if E > 1 else np.zeros(0, dtype=np.int64)
    if E > 5:
        cuts[2] = cuts[1]   # an expert without rows
    off = np.concatenate([[0], cuts, [rows - 3]]).astype(np.int32)   # three rows at the end are nobody's
    W = R.up(H, 128)
    x, w = operand(rng, rows, W), operand(rng, E, N, W)
    x[:, H:], w[:, :, H:] = 0, 0
    x, w = f8(x).cuda(), f8(w).cuda()
    xs = dev(rng.integers(120, 135, (rows, R.up(H, 512) // 128), dtype=np.uint8))
    ws = dev(rng.integers(115, 130, (E, R.up(N, 128) // 128, R.up(H, 512) // 128), dtype=np.uint8))
    out = torch.full((rows, N), -77.0, dtype=dtype, device="cuda")
    B.hm_expert_matmul(x, xs, w, ws, dev(off), out)
    a = gpu_values(x, xs[:, :W // 128])
    assert (out[rows - 3:] == -77).all()
    for e in range(E):
        r = slice(off[e], off[e + 1])
        if off[e] < off[e + 1]:
            b = gpu_values(w[e], ws[e].repeat_interleave(128, dim=0)[:N, :W // 128])
            same_in_every_patch(out[r], a[r], b, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("counts,N,H", [([700, 0, 129, 1500], 2100, 2000), ([300, 1, 250], 1000, 1541), ([128 * 11], 2050, 1030), ([5, 600], 4100, 3900)])
def test_weights_gradient_of_many(counts, N, H, dtype):
    rng = np.random.default_rng(N)
    off, E = offsets_of(counts), len(counts)
    rows = int(off[-1])
    blocks = rows // 128 + E
    gy, x = operand(rng, N, 128 * blocks), operand(rng, H, 128 * blocks)
    for e in range(E):
        first = 128 * (off[e] // 128 + e)
        for q in (gy, x):
            q[:, first + counts[e]:first + R.up(counts[e], 128)] = 0
    gy, x = f8(gy).cuda(), f8(x).cuda()
    gs, xs = dev(rng.integers(120, 135, (blocks, N), dtype=np.uint8)), dev(rng.integers(115, 130, (blocks, H), dtype=np.uint8))
    dw = torch.full((E, N, H), -77.0, dtype=dtype, device="cuda")
    B.hm_expert_matmul_dw(gy, gs, x, xs, dev(off), rows, dw)
    a, b = gpu_values(gy, gs.t()), gpu_values(x, xs.t())
    for e in range(E):
        first = 128 * (off[e] // 128 + e)
        k = slice(first, first + R.up(counts[e], 128))
        if counts[e] == 0:
            assert not dw[e].any()
            continue
        same_in_every_patch(dw[e], a[:, k].contiguous(), b[:, k].contiguous(), dtype)


def test_every_call_is_taken_by_the_native_half(monkeypatch):
    """Dense tensors on the current stream do not go through ctypes; what is out of the ordinary does, with the same result."""
    B.lib()

    class Recorder:
        calls = []

        def __getattr__(self, name):
            def call(*args):
                rc = getattr(native, name)(*args)
                self.calls.append((name, rc is not None))
                return rc
            return call

    native, rec = B._native, Recorder()
    monkeypatch.setattr(B, "_native", rec)
    T, E, K, H, N = 40, 16, 4, 96, 72
    router = B.Router(E, K)
    logits, ids, w = torch.randn((T, E), device="cuda"), torch.empty((T, K), dtype=torch.int32, device="cuda"), torch.empty((T, K), device="cuda")
    plan = B.alloc_plan(T, K, E, 1, 1, B.HM_DEDUP_NONE, num_dest=E)
    B.hm_route(logits, router, ids, w)
    B.hm_plan_mapped(ids, w, torch.arange(E, dtype=torch.int32, device="cuda"), E, False, plan=plan)
    off, rows = plan.dest_offset, T * K
    x, y, gout, master = (torch.randn(s, device="cuda") for s in ((rows, H), (rows, N), (T, N), (E, N, H)))
    both = {}
    for stream in (None, torch.cuda.current_stream()):
        x8, xt, yt = B.alloc_rows8(rows, H), B.alloc_columns8(rows, E, H), B.alloc_columns8(rows, E, N)
        w8, wt = B.alloc_weights8(E, N, H), B.alloc_weights8(E, H, N)
        for t in (*xt, *yt):
            t.view(torch.uint8).zero_()
        out, dw, gw, gl = torch.empty((rows, N), device="cuda"), torch.empty((E, N, H), device="cuda"), torch.empty((T, K), device="cuda"), torch.empty((T, E), device="cuda")
        rec.calls.clear()
        B.hm_route(logits, router, ids, w, stream=stream)
        B.hm_quantize_rows(x, *x8, stream=stream)
        B.hm_quantize_columns(x, off, *xt, stream=stream)
        B.hm_quantize_columns(y, off, *yt, stream=stream)
        B.hm_quantize_weights(master, *w8, *wt, stream=stream)
        B.hm_expert_matmul(*x8, *w8, off, out, stream=stream)
        B.hm_expert_matmul_dw(*yt, *xt, off, rows, dw, stream=stream)
        B.hm_combine_weight_grad(gout, y, plan, gw, stream=stream)
        B.hm_route_backward(logits, router, ids, gw, gl, stream=stream)
        both[stream] = [t.clone().view(torch.uint8) for t in (ids, w, *x8, *xt, *w8, *wt, out, dw, gw, gl)]
        if stream is None:
            assert len(rec.calls) == 9 and all(taken for _, taken in rec.calls), rec.calls
            assert {"hm_" + name for name, _ in rec.calls} == set(B._NATIVE_LAYER)
        else:
            assert not rec.calls
    assert all(torch.equal(a, b) for a, b in zip(*both.values()))


@pytest.mark.parametrize("width", [100, 300])
def test_parts_of_blocks_are_refused_before_any_launch(width, monkeypatch):
    """The native half leaves them to the Python code, which raises."""
    B.lib()
    taken, native = [], B._native

    class Recorder:
        def __getattr__(self, name):
            return lambda *args: taken.append(getattr(native, name)(*args))

    monkeypatch.setattr(B, "_native", Recorder())
    e8 = lambda *shape: torch.zeros(shape, dtype=F8, device="cuda")
    byte = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device="cuda")
    operands = (e8(4, width), byte(4, B.scale8_bytes(width)), e8(2, 8, width), byte(2, 1, B.scale8_bytes(width)))
    off, out = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros((4, 8), device="cuda")
    for stream in (None, torch.cuda.current_stream()):
        with pytest.raises(ValueError, match="whole blocks"):
            B.hm_expert_matmul(*operands, off, out, stream=stream)
    assert taken == [None]


def test_few_rows_of_more_strips_than_workgroups():
    """As many columns that a launch has no workgroups for strips of 16 x 16, weights beyond 2^32 bytes: sums in 32 bits all the same."""
    E, N, H = 1024, 131077, 128
    rows = 2 * E
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    w8 = torch.randint(0, 0x7F, (E, N, H), generator=g, dtype=torch.uint8, device="cuda").view(F8)
    x8 = torch.randint(0, 0x7F, (rows, H), generator=g, dtype=torch.uint8, device="cuda").view(F8)
    xs = torch.randint(120, 135, (rows, 4), generator=g, dtype=torch.uint8, device="cuda")
    ws = torch.randint(115, 130, (E, R.up(N, 128) // 128, 4), generator=g, dtype=torch.uint8, device="cuda")
    out, half = (torch.full((rows, N), -77.0, dtype=dtype, device="cuda") for dtype in (torch.float32, torch.bfloat16))
    for o in (out, half):
        B.hm_expert_matmul(x8, xs, w8, ws, dev(np.arange(0, rows + 1, 2, dtype=np.int32)), o)
    assert torch.equal(half, out.to(torch.bfloat16))
    a = gpu_values(x8, xs[:, :1])
    for e in (0, 1, 500, 1023):
        b = gpu_values(w8[e], ws[e].repeat_interleave(128, dim=0)[:N, :1])
        want = a[2 * e:2 * e + 2] @ b.t().contiguous()   # of numbers of one sign, so that a sum's error is its own: 2^-24 for each of 128 terms
        assert ((out[2 * e:2 * e + 2].double() - want).abs() <= 136 * 2.0 ** -24 * want).all(), e


def test_results_do_not_depend_on_what_ran_before():
    """The same call into poisoned outputs: the same bits."""
    rng = np.random.default_rng(8)
    off = dev(offsets_of([500, 0, 12, 300]))
    x, xs = f8(operand(rng, 812, 1024)).cuda(), dev(rng.integers(120, 130, (812, 8), dtype=np.uint8))
    w, ws = f8(operand(rng, 4, 384, 1024)).cuda(), dev(rng.integers(120, 130, (4, 3, 8), dtype=np.uint8))
    for dtype in DTYPES:
        outs = [torch.full((812, 384), fill, dtype=dtype, device="cuda") for fill in (1.0, float("nan"))]
        for o in outs:
            B.hm_expert_matmul(x, xs, w, ws, off, o)
        assert torch.equal(*[o.view(torch.uint8) for o in outs])


def test_replayed_in_a_graph():
    rng = np.random.default_rng(6)
    rows, E, N, H = 700, 4, 256, 512
    off = dev(offsets_of([300, 0, 150, 250]))
    x = torch.empty((rows, H), device="cuda")
    w = B.hm_quantize_weights(torch.randn((E, N, H), device="cuda"), *B.alloc_weights8(E, N, H))
    q, qt, y = B.alloc_rows8(rows, H), B.alloc_columns8(rows, E, H), torch.empty((rows, N), dtype=torch.bfloat16, device="cuda")
    dw = torch.empty((E, H, H), device="cuda")

    def calls():
        B.hm_quantize_rows(x, *q)
        B.hm_quantize_columns(x, off, *qt)
        B.hm_expert_matmul(*q, *w, off, y)
        B.hm_expert_matmul_dw(*qt, *qt, off, rows, dw)

    x.normal_()
    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        x.normal_()
        calls()
        want = [y.clone(), dw.clone()]
        y.fill_(7)
        dw.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(dw, want[1])
