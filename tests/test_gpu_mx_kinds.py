"""Every kernel of the microscaled product, in each of its three forms (exact float32 results of MXFP8 rows, bf16
results of MXFP8 rows, MXFP4 rows), at sizes where its rings of copies wrap several times and M, N and K end inside a
tile: sums, the exact form's products, high scale codes and NaN.  The sizes follow the library's own choice, which a
CPU test compares with what they are meant for."""
import sys

import pytest
import torch

import mx_reference as R
from paper_2608_26574_amd import dard

gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
FORMS = [(dard.MX_FP8, F32), (dard.MX_FP8, BF16), (dard.MX_FP4, F32)]
E2M1 = [0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6]

# kernel (rows, columns, parts of K; 0: tiles through LDS) and the sizes that take it, one for all forms or one each
KINDS = [((32, 256, 1), (1, 33010, 4512)), ((32, 256, 1), ((1030, 1030, 4512), (1030, 1030, 4512), (70, 16520, 4512))),
         ((32, 128, 4), (2100, 260, 9632)), ((32, 64, 4), (1030, 260, 9632)), ((32, 32, 8), (33, 70, 19104)),
         ((64, 256, 1), (2100, 1030, 4512)), ((64, 128, 4), (1030, 1030, 9632)),
         ((128, 256, 1), ((600, 12300, 3232), (2100, 2070, 3232), (2100, 2070, 4512))),
         ((256, 256, 0), (1030, 12300, 1696)), ((256, 256, 0), (2100, 12300, 3232))]
CASES = [(kind, *form, *(sizes if isinstance(sizes[0], int) else sizes[i])) for kind, sizes in KINDS
         for i, form in enumerate(FORMS)]
EXACT = [(k, M, N, K) for k, fmt, out, M, N, K in CASES if fmt == dard.MX_FP8 and out is F32]


def test_sizes_take_every_kernel():
    seen = set()
    for kind, fmt, out, M, N, K in CASES:
        plan = dard.dard_linear_mx_plan(fmt, M, N, K, out)
        assert plan == (*kind, int(fmt == dard.MX_FP8 and out is F32)), (kind, fmt, out, M, N, K)
        assert M % kind[0] and N % kind[1] and K % 256
        # units of 256 k that a wave takes: past the chunks of scales (8, 12 or 16 units), and stages of half
        # a unit three times round the rings of 3 or 4
        units = -(-K // 256) / max(1, kind[2])
        assert units >= {1: 13 if kind[0] == 128 else 17, 0: 6}.get(kind[2], 9)
        seen.add((kind, fmt, out))
    # every kernel that any size takes (a sweep that holds all of them)
    for fmt, out in FORMS:
        for M in (1, 20, 33, 64, 100, 200, 600, 1030, 4100):
            for N in (32, 260, 1030, 3584, 8230, 12300, 33010):
                for K in (32, 1024, 3584, 9632, 19104):
                    assert (dard.dard_linear_mx_plan(fmt, M, N, K, out)[:3], fmt, out) in seen


def test_plan_refusals():
    plan = dard.dard_linear_mx_plan
    for bad in ((2, 4, 64, 64), (0, 0, 64, 64), (0, 4, 0, 64), (0, 4, 64, 48)):
        with pytest.raises(dard.DardError):
            plan(*bad)
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        plan(0, 4, 64, 64, torch.float16)
    assert dard.lib().dard_linear_mx_plan(0, 4, 64, 64, 0, None) == -1


# ------------------------------------------------------------------ inputs, and their values in float64
def announce(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def ints(g, lo, hi, *shape):
    return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.uint8)


def packed(codes, scales):
    """The packed weights of E2M1 codes, one a byte."""
    wp = torch.full((dard.dard_packed_mx_bytes(codes.shape[0], codes.shape[1]),), 0x77, dtype=torch.uint8, device="cuda")
    dard.dard_pack_matrix_mx(stored(codes, dard.MX_FP4), scales, wp)
    return wp


def stored(codes, fmt):
    return codes if fmt == dard.MX_FP8 else codes[:, ::2] | codes[:, 1::2] << 4


def values(codes, scales, fmt):
    table = torch.tensor(E2M1 if fmt == dard.MX_FP4 else R.F8, dtype=torch.float64, device="cuda")
    return table[codes.long()] * torch.exp2(scales.double() - 127).repeat_interleave(32, 1)


def product(fmt, codes, scales, wp, N, out):
    M = codes.shape[0]
    y = torch.full((M * N + 32,), 7.0, dtype=out, device="cuda")
    dard.dard_linear_mx(fmt, stored(codes, fmt), scales, wp, y[:M * N].view(M, N))
    assert bool((y[M * N:] == 7.0).all())
    return y[:M * N].view(M, N)


def random_operands(fmt, M, N, K, seed):
    """Random finite codes, scales over eight powers of two."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = ints(g, 0, 16, M, K) if fmt == dard.MX_FP4 else ints(g, 0, 127, M, K) | ints(g, 0, 2, M, K) << 7
    return x, ints(g, 120, 128, M, K // 32), ints(g, 0, 16, N, K), ints(g, 120, 128, N, K // 32)


# ------------------------------------------------------------------ tests
@gpu
@pytest.mark.parametrize("kind,fmt,out,M,N,K", CASES)
def test_exact_sums(kind, fmt, out, M, N, K):
    """Products that are small multiples of 1/16: their sums are exact in float32 in any order, and no bit of them
    lies below what the matrix instructions keep."""
    announce("linear kinds, exact sums", kind, fmt, out, M, N, K)
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    few = torch.tensor([0, 0x30, 0x38, 0x3C, 0x40, 0x80, 0xB0, 0xB8, 0xBC, 0xC0], dtype=torch.uint8, device="cuda")   # 0 to 2
    x = ints(g, 0, 16, M, K) if fmt == dard.MX_FP4 else few[ints(g, 0, 10, M, K).long()]
    xs, w, ws = ints(g, 126, 129, M, K // 32), ints(g, 0, 16, N, K), ints(g, 126, 129, N, K // 32)
    ref = values(x, xs, fmt) @ values(w, ws, dard.MX_FP4).T
    assert torch.equal(product(fmt, x, xs, packed(w, ws), N, out), ref.float().to(out))


@gpu
@pytest.mark.parametrize("kind,M,N,K", EXACT)
def test_float32_products_are_exact(kind, M, N, K):
    """Eight neighbouring products that span 2^16, two large ones that cancel among them: the small ones count.
    All sums are multiples of u = 2^-8 below 2^24 u in any order (float32 holds them): at most 200 of a
    row's groups have a pair of +-2^8 = 2^16 u, the other products are 12 u at most."""
    announce("linear kinds, exact products", kind, M, N, K)
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    w = torch.tensor([1, 2, 9, 10], dtype=torch.uint8, device="cuda")[ints(g, 0, 4, N, K // 2).long()].repeat_interleave(2, 1)
    ws = (127 - torch.arange(N, device="cuda") % 2).to(torch.uint8)[:, None].repeat(1, K // 32)          # (a factor of
    xs = (127 + torch.arange(M, device="cuda") % 3).to(torch.uint8)[:, None].repeat(1, K // 32)          # the result)
    small = torch.tensor([0x08, 0x0C, 0x10, 0x14, 0x88, 0x8C, 0x90, 0x94], dtype=torch.uint8, device="cuda")   # 1 to 3 times 2^-6
    x = small[ints(g, 0, 8, M, K).long()].view(M, K // 8, 4, 2)
    large = torch.rand(M, K // 8, generator=g, device="cuda") < min(0.5, 80 / (K // 8))
    assert int(large.sum(1).max()) <= 200 and 200 * 2 ** 16 + 12 * K < 2 ** 24
    pair = torch.randint(0, 4, (M, K // 8), generator=g, device="cuda")
    at = large[:, :, None] & (pair[:, :, None] == torch.arange(4, device="cuda"))
    x[at] = torch.tensor([0x78, 0xF8], dtype=torch.uint8, device="cuda")                                 # 256, -256
    x = x.view(M, K)
    wv = values(w, ws, dard.MX_FP4)
    ref = (values(x, xs, dard.MX_FP8) @ wv.T).float()
    got = product(dard.MX_FP8, x, xs, packed(w, ws), N, F32)
    assert torch.equal(got, ref), float((got != ref).float().mean())
    # the test can tell: cut 13 bits below the largest, the small products of those groups would be gone
    cut = torch.where(large[:, :, None].expand(-1, -1, 8).reshape(M, K) & ~at.repeat_interleave(2, 2).view(M, K), x, 0)
    assert float(((values(cut, xs, dard.MX_FP8) @ wv.T) != 0).float().mean()) > 0.9


@gpu
@pytest.mark.parametrize("M,N,K", [(48, 512, 4096), (320, 256, 3584)])
def test_float32_error_norm(M, N, K):
    """K / 16 rounded additions, each within 2^-24 of a partial sum: at random, 2^-24 sqrt(K / 32) = 7e-7 of the
    result at most at these K (products cut 13 bits below the largest of eight leave 4.5e-6)."""
    announce("linear kinds, error norm", M, N, K)
    g = torch.Generator(device="cuda").manual_seed(K)
    x, w = torch.randn(M, K, generator=g, device="cuda"), torch.randn(N, K, generator=g, device="cuda")
    xc, xs = torch.empty(M, K, dtype=torch.uint8, device="cuda"), torch.empty(M, K // 32, dtype=torch.uint8, device="cuda")
    wc, ws = torch.empty(N, K // 2, dtype=torch.uint8, device="cuda"), torch.empty(N, K // 32, dtype=torch.uint8, device="cuda")
    dard.dard_quantize_mx(x, dard.MX_FP8, xc, xs)
    dard.dard_quantize_mx(w, dard.MX_FP4, wc, ws)
    codes = torch.stack([wc & 15, wc >> 4], -1).flatten(1)
    ref = values(xc, xs, dard.MX_FP8) @ values(codes, ws, dard.MX_FP4).T
    got = product(dard.MX_FP8, xc, xs, packed(codes, ws), N, F32).double()
    assert float((got - ref).norm() / ref.norm()) <= 2.0 ** -24 * (K / 32) ** 0.5


@gpu
@pytest.mark.parametrize("kind,M,N,K", EXACT)
def test_high_scales_stay_local(kind, M, N, K):
    """Scale codes past those of quantised float32 in one row of x and one of w: their results are right, the
    others keep their bits."""
    announce("linear kinds, high scales", kind, M, N, K)
    x, xs, w, ws = random_operands(dard.MX_FP8, M, N, K, 1)
    xs[:, 0], ws[:, -1] = 40, 40
    clean = product(dard.MX_FP8, x, xs, packed(w, ws), N, F32).clone()
    m, n = M * 2 // 3, N - 5
    xs[m, -1], ws[n, 0] = 250, 254   # (times 2^-87 of the others': in range)
    got = product(dard.MX_FP8, x, xs, packed(w, ws), N, F32)
    rest = torch.ones(M, N, dtype=torch.bool, device="cuda")
    rest[m], rest[:, n] = False, False
    assert torch.equal(got[rest], clean[rest])
    xv, wv = values(x, xs, dard.MX_FP8), values(w, ws, dard.MX_FP4)
    for p, y in ((xv[m] * wv, got[m]), (xv * wv[n], got[:, n])):
        # sums in float32 of products cut 2^-13 below the largest of eight (at most seven are)
        bound = p.abs().sum(1) * K * 2.0 ** -23 + 7 * 2.0 ** -13 * p.abs().view(p.shape[0], -1, 8).amax(-1).sum(1)
        assert bool(((y.double() - p.sum(1)).abs() <= bound).all())


@gpu
@pytest.mark.parametrize("kind,fmt,out,M,N,K", CASES)
def test_nan_stays_local(kind, fmt, out, M, N, K):
    """NaN scales in a row of x and one of w, and a NaN code in another row of x, make their results NaN and no
    others differ."""
    announce("linear kinds, NaN", kind, fmt, out, M, N, K)
    x, xs, w, ws = random_operands(fmt, M, N, K, 2)
    clean = product(fmt, x, xs, packed(w, ws), N, out).clone()
    assert bool(torch.isfinite(clean).all())
    xs[M - 1, -1], ws[N // 2, 3] = 255, 255
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[M - 1], bad[:, N // 2] = True, True
    if fmt == dard.MX_FP8:
        x[0, K - 1] = 0xFF
        bad[0] = True
    got = product(fmt, x, xs, packed(w, ws), N, out)
    assert bool(torch.isnan(got[bad]).all())
    assert torch.equal(got[~bad], clean[~bad])
