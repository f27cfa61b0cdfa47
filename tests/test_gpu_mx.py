"""The microscaled quantisation, norm and product against plain float64 forms
(tests/mx_reference.py): every code byte and scale must be equal -- the roundings
are decided in exact arithmetic or in 64 bits --, and products lie within the
bound that the arithmetic gives."""
import sys

import numpy as np
import pytest
import torch

import mx_reference as R
from paper_2608_26574_amd import dard

pytestmark = pytest.mark.gpu

FORMATS = [dard.MX_FP8, dard.MX_FP4]
GUARD = 0xA5


def announce(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def f64(t):
    return t.double().cpu().numpy()


def guarded(*shape):
    """A uint8 buffer [*shape] followed by 64 guard bytes: (view, whole)."""
    n = int(np.prod(shape))
    t = torch.full((n + 64,), GUARD, dtype=torch.uint8, device="cuda")
    return t[:n].view(*shape), t


def code_shape(rows, K, fmt):
    return (rows, K if fmt == dard.MX_FP8 else K // 2)


def quantized(x, fmt):
    """Codes and scales of device tensor x by the library, guards checked."""
    rows, K = x.shape
    codes, wc = guarded(*code_shape(rows, K, fmt))
    scales, ws = guarded(rows, K // 32)
    dard.dard_quantize_mx(x, fmt, codes, scales)
    torch.cuda.synchronize()
    assert bool((wc[codes.numel():] == GUARD).all()) and bool((ws[scales.numel():] == GUARD).all())
    return codes, scales


def check_codes(codes, scales, x, fmt):
    c, s = R.quantize(x, fmt)
    assert np.array_equal(scales.cpu().numpy(), s)
    assert np.array_equal(codes.cpu().numpy(), R.pack(c, fmt))


def hard_rows(rows, K, seed):
    """Rows with blocks of every kind: wide ranges, zeros, subnormals, the largest floats, ties."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, K)) * np.exp2(rng.integers(-30, 30, (rows, K // 32)).repeat(32, 1))
    kind = rng.integers(0, 8, (rows, K // 32))
    for i, j in zip(*np.nonzero(kind < 6)):
        b = slice(32 * j, 32 * j + 32)
        k = kind[i, j]
        if k == 0:
            x[i, b] = 0.0
        elif k == 1:
            x[i, b] = rng.integers(-60, 61, 32) * 2.0 ** -149      # subnormal float32
        elif k == 2:
            x[i, b] = rng.choice([-1, 1], 32) * 2.0 ** 127 * rng.choice([1, 1.25, 1.5, 1.875], 32)
        elif k == 3:
            x[i, b] = rng.integers(-64, 65, 32) / 64 * 6           # ties of both formats
        elif k == 4:
            x[i, b] = np.exp2(rng.integers(-20, 1, 32))            # powers of two: block maxima on a border
        else:
            x[i, b] = -0.0
    return x


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,K,extra", [(1, 32, 0), (3, 96, 5), (70, 1056, 0), (257, 4096, 3)])
def test_quantize(fmt, dtype, rows, K, extra):
    announce("quantize", fmt, dtype, rows, K, extra)
    wide = torch.from_numpy(hard_rows(rows, K + 32, rows + K)).to(dtype).cuda()[:, :K + extra]
    x = wide.contiguous()[:, :K] if extra else wide[:, :K].contiguous()
    codes, scales = quantized(x, fmt)
    check_codes(codes, scales, f64(x), fmt)
    back = torch.full((rows, K + 7), 3.0, dtype=dtype, device="cuda")
    dard.dard_dequantize_mx(fmt, codes, scales, back[:, :K])
    ref = R.values(*R.quantize(f64(x), fmt), fmt)
    # (E4M3 times 2^-127 has bits below bf16's smallest subnormal: rounded once)
    ref = torch.from_numpy(ref).float().to(dtype) if dtype == torch.bfloat16 else torch.from_numpy(ref).float()
    assert torch.equal(back[:, :K].cpu(), ref)
    assert bool((back[:, K:] == 3.0).all())


@pytest.mark.parametrize("fmt", FORMATS)
def test_quantize_every_bf16(fmt):
    announce("quantize every bf16", fmt)
    bits = np.arange(65536, dtype=np.uint32)
    bits = bits[((bits >> 7) & 255) != 255].reshape(-1, 32)   # finite values
    rng = np.random.default_rng(1)
    bits = bits.reshape(-1)[rng.permutation(bits.size)].reshape(-1, 32)
    x = dev((bits << 16).astype(np.uint32).view(np.float32)).bfloat16()
    codes, scales = quantized(x, fmt)
    check_codes(codes, scales, f64(x), fmt)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_quantize_not_finite(fmt, bad):
    announce("quantize not finite", fmt, bad)
    x = np.random.default_rng(2).standard_normal((4, 128)).astype(np.float32)
    x[1, 40] = x[3, 0] = x[3, 127] = bad
    codes, scales = quantized(dev(x), fmt)
    check_codes(codes, scales, x.astype(np.float64), fmt)
    y = torch.zeros(4, 128, device="cuda")
    dard.dard_dequantize_mx(fmt, codes, scales, y)
    nan = torch.isnan(y).cpu().numpy().reshape(4, 4, 32)
    want = np.zeros((4, 4), bool)
    want[1, 1] = want[3, 0] = want[3, 3] = True
    assert np.array_equal(nan, np.broadcast_to(want[..., None], nan.shape))


@pytest.mark.parametrize("fmt", FORMATS)
def test_dequantize_every_code_and_scale(fmt):
    announce("dequantize all", fmt)
    scales = np.arange(256, dtype=np.uint8).repeat(8)[:, None]
    one = np.arange(256, dtype=np.uint8).reshape(8, 32) if fmt == dard.MX_FP8 else (np.arange(256).reshape(8, 32) % 16).astype(np.uint8)
    codes = np.tile(one, (256, 1))
    x = torch.empty(2048, 32, device="cuda")
    dard.dard_dequantize_mx(fmt, dev(R.pack(codes, fmt)), dev(scales), x)
    with np.errstate(over="ignore"):
        ref = R.values(codes, scales, fmt).astype(np.float32)
    assert np.array_equal(x.cpu().numpy(), ref, equal_nan=True)


# d: one block, part of a wave, whole waves, an odd number of blocks, several chunks a thread, the largest
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,d,delta,gain", [(1, 32, "f32", "f32"), (5, 256, None, "bf16"), (64, 4096, "f32", "bf16"),
                                               (7, 2080, "bf16", "f32"), (33, 3584, "bf16", "bf16"),
                                               (3, 8192, "f32", "f32"), (2, 6176, None, "f32"), (700, 1024, "bf16", "bf16")])
def test_resid_norm(fmt, rows, d, delta, gain):
    announce("resid norm", fmt, rows, d, delta, gain)
    g = torch.Generator(device="cuda").manual_seed(d + rows)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}
    h = torch.randn(rows, d, generator=g, device="cuda") * 3
    h *= 1 + 30 * (torch.rand(d, generator=g, device="cuda") < 0.01)
    dl = None if delta is None else torch.randn(rows, d, generator=g, device="cuda").to(dt[delta])
    gn = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dt[gain])
    if rows > 2:
        h[1] = 0.0
        if dl is not None:
            dl[1] = 0.0
    want_h, y = R.norm(h.cpu().numpy(), None if dl is None else dl.float().cpu().numpy(), gn.float().cpu().numpy(), 1e-5)
    codes, wc = guarded(*code_shape(rows, d, fmt))
    scales, ws = guarded(rows, d // 32)
    dard.dard_resid_norm_mx(h, gn, 1e-5, fmt, codes, scales, delta=dl)
    torch.cuda.synchronize()
    assert np.array_equal(h.cpu().numpy(), want_h)
    check_codes(codes, scales, y, fmt)   # (64-bit sums differ by 2^-50: no value of these inputs lies that near a border)
    assert bool((wc[codes.numel():] == GUARD).all()) and bool((ws[scales.numel():] == GUARD).all())


def test_resid_norm_not_finite():
    announce("resid norm not finite")
    h = torch.randn(4, 512, device="cuda")
    h[1, 7], h[2, 500] = float("inf"), float("nan")
    codes, scales = torch.empty(4, 512, dtype=torch.uint8, device="cuda"), torch.empty(4, 16, dtype=torch.uint8, device="cuda")
    dard.dard_resid_norm_mx(h, torch.ones(512, device="cuda"), 0.0, dard.MX_FP8, codes, scales)
    s = scales.cpu().numpy()
    # the infinity's row: 0 everywhere but inf * 0 = NaN in its own block
    assert (s[2] == 255).all() and (s[1, 0] == 255) and (s[[0, 3]] != 255).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [96, 512, 4128])
def test_resid_norm_rows_not_finite(fmt, d):
    """An infinity (one that the addition makes, too) leaves NaN in its own block and zeros in the others of
    its row, a NaN or, without eps, a row of zeros NaN everywhere; other rows keep their values."""
    announce("resid norm rows not finite", fmt, d)
    g = torch.Generator(device="cuda").manual_seed(d)
    h, dl = torch.randn(6, d, generator=g, device="cuda"), torch.randn(6, d, generator=g, device="cuda")
    h[1, 40], h[2, d - 1] = float("inf"), float("nan")
    h[3, 70] = dl[3, 70] = 3e38
    h[4] = dl[4] = 0.0
    gn = torch.ones(d, device="cuda")
    with np.errstate(over="ignore"):
        want_h, y = R.norm(h.cpu().numpy(), dl.cpu().numpy(), gn.cpu().numpy(), 0.0)
    codes = torch.empty(code_shape(6, d, fmt), dtype=torch.uint8, device="cuda")
    scales = torch.empty(6, d // 32, dtype=torch.uint8, device="cuda")
    dard.dard_resid_norm_mx(h, gn, 0.0, fmt, codes, scales, delta=dl)
    assert np.array_equal(h.cpu().numpy(), want_h, equal_nan=True)
    s = scales.cpu().numpy()
    nan = np.zeros_like(s, bool)
    nan[1, 1] = nan[3, 2] = nan[2] = nan[4] = True
    assert np.array_equal(s == 255, nan) and (s[[1, 3]][~nan[[1, 3]]] == 0).all()
    check_codes(codes, scales, y, fmt)


def mx_rows(rows, K, fmt, seed, spread=2.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, K)) * np.exp2(rng.uniform(-spread, spread, (rows, K)))
    c, s = R.quantize(x, fmt)
    return c, s, R.values(c, s, fmt)


def run_linear(xc, xs, fmt, wc, ws, N, out):
    M = xc.shape[0]
    K = 32 * xs.shape[1]
    wp = torch.full((dard.dard_packed_mx_bytes(N, K),), 0x77, dtype=torch.uint8, device="cuda")
    dard.dard_pack_matrix_mx(dev(R.pack(wc, R.FP4)), dev(ws), wp)
    y = torch.full((M * N + 32,), 7.0, dtype=out, device="cuda")
    room = torch.full((dard.dard_linear_mx_workspace_bytes(fmt, M, N, K) // 4,), float("nan"), device="cuda")
    dard.dard_linear_mx(fmt, dev(R.pack(xc, fmt)), dev(xs), wp, y[:M * N].view(M, N), ws=room)
    torch.cuda.synchronize()
    assert bool((y[M * N:] == 7.0).all())
    return y[:M * N].view(M, N)


# rows and columns inside, at and past a tile; K of one block, inside a unit of 256, odd numbers of blocks, long
SHAPES = [(1, 1, 32), (1, 33, 96), (2, 16, 256), (31, 40, 288), (33, 64, 512), (64, 100, 992), (65, 31, 1024),
          (97, 257, 320), (130, 96, 2080), (3, 4096, 64), (1, 64, 12288), (64, 512, 4096), (256, 260, 768), (300, 520, 1056)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_linear(fmt, out, M, N, K):
    announce("linear", fmt, out, M, N, K)
    xc, xs, x = mx_rows(M, K, fmt, M + N)
    wc, ws, w = mx_rows(N, K, R.FP4, K)
    got = f64(run_linear(xc, xs, fmt, wc, ws, N, out))
    ref = x @ w.T
    bound = np.concatenate([R.product_bound(x, w[i:i + 64], scaled=True) for i in range(0, N, 64)], 1)
    if out == torch.bfloat16:
        bound = bound + (np.abs(ref) + bound) * 2.0 ** -8
    assert np.all(np.abs(got - ref) <= bound + 1e-30), float(np.max(np.abs(got - ref) / (bound + 1e-30)))


# as ordinary data gives them: the norm of the error
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K", [(48, 512, 4096), (320, 256, 3584)])
def test_linear_error_norm(fmt, M, N, K):
    announce("linear error norm", fmt, M, N, K)
    xc, xs, x = mx_rows(M, K, fmt, 5, spread=0.0)
    wc, ws, w = mx_rows(N, K, R.FP4, 6, spread=0.0)
    got, ref = f64(run_linear(xc, xs, fmt, wc, ws, N, torch.float32)), x @ w.T
    # float32's own: partial sums of the size of the result, K / 64 of them rounded or cut at 2^-23
    assert np.linalg.norm(got - ref) <= 1e-5 * np.linalg.norm(ref)


# every kernel and both sides of its choice: rows per workgroup 32 to 256, K split over 1 to 8 groups of waves,
# chunks of scales that are refilled, K that ends inside a unit
CHOICES = [(1, 70, 1056), (1, 8230, 544), (1, 16520, 800), (33, 33010, 32), (33, 8230, 800), (1000, 12300, 32),
           (1, 16520, 32), (100, 33010, 32), (5, 33010, 6240), (5, 16520, 12320), (5, 8230, 33056), (64, 520, 33056),
           (40, 33010, 6240), (40, 8230, 33056), (100, 33010, 6240), (600, 8230, 4128), (2050, 4130, 2080), (1030, 33010, 288), (33, 16520, 12320), (1, 70, 3360)]


@pytest.mark.parametrize("M,N,K", CHOICES)
def test_linear_exact_sums(M, N, K):
    """Values whose products are small multiples of 1/16: their sums are exact in float32 in any order, and
    within the bits that the matrix instructions keep."""
    announce("linear exact sums", M, N, K)
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    def ints(hi, *shape):
        return torch.randint(0, hi, shape, generator=g, device="cuda", dtype=torch.uint8)
    e2m1 = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    e4m3 = torch.tensor([0, 0x30, 0x38, 0x3C, 0x40, 0x80, 0xB0, 0xB8, 0xBC, 0xC0], device="cuda", dtype=torch.uint8)
    v4m3 = torch.tensor([0, .5, 1, 1.5, 2, 0, -.5, -1, -1.5, -2], device="cuda")
    def times(v, sc):
        return v * torch.exp2(sc.float() - 127).repeat_interleave(32, 1)
    wi, ws = ints(16, N, K), 126 + ints(3, N, K // 32)
    wp = torch.empty(dard.dard_packed_mx_bytes(N, K), dtype=torch.uint8, device="cuda")
    dard.dard_pack_matrix_mx(wi[:, ::2] | wi[:, 1::2] << 4, ws, wp)
    w = times(e2m1[wi.long()], ws).double()
    xs = 126 + ints(3, M, K // 32)
    for fmt in FORMATS:
        xi = ints(10 if fmt == R.FP8 else 16, M, K).long()
        codes = e4m3[xi] if fmt == R.FP8 else (xi[:, ::2] | xi[:, 1::2] << 4).to(torch.uint8)
        x = times((v4m3 if fmt == R.FP8 else e2m1)[xi], xs).double()
        ref = x @ w.T
        for out in (torch.float32, torch.bfloat16):
            y = torch.full((M * N + 32,), 7.0, dtype=out, device="cuda")
            dard.dard_linear_mx(fmt, codes, xs, wp, y[:M * N].view(M, N))
            assert bool((y[M * N:] == 7.0).all())
            assert torch.equal(y[:M * N].view(M, N), ref.to(torch.float32).to(out)), (fmt, out)


@pytest.mark.parametrize("M,N,K", [(40, 100, 4096), (40, 8230, 800), (300, 33010, 96)])
def test_linear_high_scales_stay_local(M, N, K):
    """Scale codes past those of quantised float32 in one row of x and one of w: their results are right, the
    others keep their bits."""
    announce("linear high scales", M, N, K)
    xc, xs, _ = mx_rows(M, K, R.FP8, 1)
    wc, ws, _ = mx_rows(N, K, R.FP4, 2)
    xs[:, 0], ws[:, -1] = 40, 40
    clean = run_linear(xc, xs, R.FP8, wc, ws, N, torch.float32).cpu().numpy()
    m, n = M - 3, N - 5
    xs[m, -1], ws[n, 0] = 250, 254   # (times 2^-87 of the others': in range)
    got = run_linear(xc, xs, R.FP8, wc, ws, N, torch.float32).cpu().numpy()
    rest = np.ones((M, N), bool)
    rest[m], rest[:, n] = False, False
    assert np.array_equal(got[rest], clean[rest])
    x, w = R.values(xc, xs, R.FP8), R.values(wc, ws, R.FP4)
    for a, b, y in ((x[m:m + 1], w, got[m:m + 1]), (x, w[n:n + 1], got[:, n:n + 1])):
        assert np.all(np.abs(y.astype(np.float64) - a @ b.T) <= R.product_bound(a, b, scaled=True))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K", [(5, 70, 512), (70, 70, 288), (280, 300, 512)])
def test_linear_nan_blocks(fmt, M, N, K):
    announce("linear nan blocks", fmt, M, N, K)
    xc, xs, x = mx_rows(M, K, fmt, 1)
    wc, ws, w = mx_rows(N, K, R.FP4, 2)
    clean = run_linear(xc, xs, fmt, wc, ws, N, torch.float32).cpu().numpy()
    xs[M - 2, -1] = 255
    ws[3, 0] = 255
    got = run_linear(xc, xs, fmt, wc, ws, N, torch.float32).cpu().numpy()
    bad = np.zeros((M, N), bool)
    bad[M - 2], bad[:, 3] = True, True
    assert np.isnan(got[bad]).all()
    assert np.array_equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("M,N,K", [(5, 70, 512), (40, 8230, 288), (300, 33010, 96)])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_linear_nan_codes(M, N, K, out):
    """An E4M3 NaN code makes its row NaN and nothing else."""
    announce("linear nan codes", M, N, K, out)
    xc, xs, _ = mx_rows(M, K, R.FP8, 1)
    wc, ws, _ = mx_rows(N, K, R.FP4, 2)
    clean = run_linear(xc, xs, R.FP8, wc, ws, N, out)
    xc[M - 2, K - 1], xc[0, 3] = 0x7F, 0xFF
    got = run_linear(xc, xs, R.FP8, wc, ws, N, out)
    rest = torch.ones(M, dtype=torch.bool)
    rest[[0, M - 2]] = False
    assert bool(torch.isnan(got[~rest]).all())
    assert torch.equal(got[rest], clean[rest])


def test_linear_scale_extremes():
    announce("linear scale extremes")
    M, N, K = 4, 32, 64
    xc, xs, _ = mx_rows(M, K, R.FP8, 1)
    wc, ws, _ = mx_rows(N, K, R.FP4, 2)
    xs[:], ws[:] = 0, 190          # 2^-127 times 2^63
    xs[1], ws[1::2] = 254, 20      # 2^127 times 2^-107
    x, w = R.values(xc, xs, R.FP8), R.values(wc, ws, R.FP4)
    got, ref = f64(run_linear(xc, xs, R.FP8, wc, ws, N, torch.float32)), x @ w.T
    ok = np.abs(ref) < 3e38
    bound = R.product_bound(x, w, scaled=True) + 2.0 ** -149
    assert np.all(np.abs(got - ref)[ok] <= bound[ok])


def test_linear_repeats():
    """The same call twice gives the same bits (sums in a fixed order), also next to a call on another stream."""
    announce("linear repeats")
    xc, xs, _ = mx_rows(20, 4096, R.FP8, 3)
    wc, ws, _ = mx_rows(256, 4096, R.FP4, 4)
    wp = torch.empty(dard.dard_packed_mx_bytes(256, 4096), dtype=torch.uint8, device="cuda")
    dard.dard_pack_matrix_mx(dev(R.pack(wc, R.FP4)), dev(ws), wp)
    codes, scales = dev(xc), dev(xs)
    n = dard.dard_linear_mx_workspace_bytes(dard.MX_FP8, 20, 256, 4096)
    ys = [torch.empty(20, 256, device="cuda") for _ in range(6)]
    rooms = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i, y in enumerate(ys):
        with torch.cuda.stream(streams[i % 2]):
            dard.dard_linear_mx(dard.MX_FP8, codes, scales, wp, y, ws=rooms[i % 2])
    torch.cuda.synchronize()
    for y in ys[1:]:
        assert torch.equal(y, ys[0])
