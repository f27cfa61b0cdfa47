"""Host-side refusals of the microscaled entry points (nothing is launched, no
GPU is needed), their sizes, and the plain forms that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

import mx_reference as R
from paper_2608_26574_amd import dard

P = ctypes.c_void_p(0x1000)      # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1001)
BIG = 1 << 40


def test_quantize_refusals():
    L = dard.lib()
    q = L.dard_quantize_mx
    assert q(1, None, 64, 2, 64, 0, P, P, None) == -1
    assert q(1, P, 64, 2, 64, 0, None, P, None) == -1
    assert q(1, P, 64, 2, 64, 0, P, None, None) == -1
    assert q(2, P, 64, 2, 64, 0, P, P, None) == -1 and b"dtype" in L.dard_last_error()
    assert q(1, P, 64, 2, 64, 2, P, P, None) == -1 and b"format" in L.dard_last_error()
    assert q(1, P, 64, 0, 64, 0, P, P, None) == -2
    assert q(1, P, 64, 2, 0, 0, P, P, None) == -2
    assert q(1, P, 64, 2, 48, 0, P, P, None) == -2
    assert q(1, P, 63, 2, 64, 0, P, P, None) == -2                   # rows would overlap
    assert q(1, P, 8192, 2 ** 31 - 1, 8192, 0, P, P, None) == -2
    assert q(1, P, 64, 2, 64, 0, ctypes.c_void_p(0x1008), P, None) == -1 and b"16-byte" in L.dard_last_error()
    assert q(1, ODD, 64, 2, 64, 0, P, P, None) == -1
    assert L.dard_dequantize_mx(5, P, P, 2, 64, 1, P, 64, None) == -1
    assert L.dard_dequantize_mx(0, P, P, 2, 64, 1, P, 32, None) == -2


def test_resid_norm_refusals():
    L = dard.lib()
    f = L.dard_resid_norm_mx
    assert f(None, 0, P, 0, P, 1e-5, 4, 64, 0, P, P, None) == -1
    assert f(P, 0, P, 0, None, 1e-5, 4, 64, 0, P, P, None) == -1
    assert f(P, 7, P, 0, P, 1e-5, 4, 64, 0, P, P, None) == -1
    assert f(P, 0, P, 2, P, 1e-5, 4, 64, 0, P, P, None) == -1
    assert f(P, 0, P, 0, P, -1.0, 4, 64, 0, P, P, None) == -1
    assert f(P, 0, P, 0, P, float("nan"), 4, 64, 0, P, P, None) == -1
    assert f(P, 0, P, 0, P, 1e-5, 0, 64, 0, P, P, None) == -2
    assert f(P, 0, P, 0, P, 1e-5, 4, 72, 0, P, P, None) == -2
    assert f(P, 0, P, 0, P, 1e-5, 4, 8224, 0, P, P, None) == -2
    assert f(P, 0, ctypes.c_void_p(0x1002), 0, P, 1e-5, 4, 64, 0, P, P, None) == -1


def test_product_refusals_and_sizes():
    L = dard.lib()
    # codes of 32-row, 256-k blocks at half a byte a value, a scale byte per 32
    assert L.dard_packed_mx_bytes(4096, 4096) == 4096 * 4096 // 2 + 4096 * 4096 // 32
    assert L.dard_packed_mx_bytes(33, 32) == 64 * 256 // 2 + 64 * 256 // 32
    assert L.dard_packed_mx_bytes(0, 64) == 0 and L.dard_packed_mx_bytes(64, 40) == 0
    assert L.dard_packed_mx_bytes(1 << 20, 1 << 13) == 0 and b"2 GiB" in L.dard_last_error()
    with pytest.raises(dard.DardError):
        dard.dard_packed_mx_bytes(64, 40)
    assert L.dard_pack_matrix_mx(None, P, 64, 64, P, None) == -1
    assert L.dard_pack_matrix_mx(P, P, 64, 65, P, None) == -2
    assert L.dard_pack_matrix_mx(ctypes.c_void_p(0x1004), P, 64, 64, P, None) == -1
    assert L.dard_linear_mx_workspace_bytes(9, 4, 64, 64) == 0
    assert L.dard_linear_mx_workspace_bytes(0, 0, 64, 64) == 0
    f = L.dard_linear_mx
    assert f(3, P, P, 4, 64, P, 64, 0, P, P, BIG, None) == -1
    assert f(0, P, P, 4, 64, P, 64, 2, P, P, BIG, None) == -1
    assert f(0, None, P, 4, 64, P, 64, 0, P, P, BIG, None) == -1
    assert f(0, P, P, 0, 64, P, 64, 0, P, P, BIG, None) == -2
    assert f(0, P, P, 4, 48, P, 64, 0, P, P, BIG, None) == -2
    assert f(0, P, P, 4, 64, P, 0, 0, P, P, BIG, None) == -2
    assert f(0, ctypes.c_void_p(0x1008), P, 4, 64, P, 64, 0, P, P, BIG, None) == -1
    assert f(0, P, P, 4, 64, P, 64, 0, ctypes.c_void_p(0x1002), P, BIG, None) == -1
    need = L.dard_linear_mx_workspace_bytes(0, 1, 4096, 12288)
    if need:
        assert f(0, P, P, 1, 12288, P, 4096, 0, P, P, need - 1, None) == -5
        assert f(0, P, P, 1, 12288, P, 4096, 0, P, None, 0, None) == -5


def test_cache_refusals():
    L = dard.lib()
    def w(dtype=1, k=P, v=P, ld=256, b=1, n=4, H=2, dh=128, pos=0, cap=64, kc=P, ks=P, vc=P, vs=P):
        return L.dard_kv_write_mx(dtype, k, v, ld, b, n, H, dh, pos, None, cap, kc, ks, vc, vs, None)
    def r(dtype=1, k=P, v=P, ld=256, b=1, n=4, H=2, dh=128, pos=0, cap=64, kc=P, ks=P, vc=P, vs=P):
        return L.dard_kv_read_mx(kc, ks, vc, vs, cap, b, n, H, dh, pos, None, dtype, k, v, ld, None)
    for f in (w, r):
        assert f(dtype=2) == -1 and f(k=None) == -1 and f(v=None) == -1 and f(kc=None) == -1 and f(vs=None) == -1
        assert f(dh=96) == -2 and f(cap=40) == -2 and f(n=0) == -2 and f(pos=-1) == -2 and f(pos=61) == -2
        assert f(n=65) == -2 and f(ld=255) == -2 and f(b=0) == -2 and f(H=0) == -2
        assert f(kc=ctypes.c_void_p(0x1008)) == -1 and f(ks=ctypes.c_void_p(0x1004)) == -1 and f(k=ODD) == -1
        assert f(pos=2 ** 31 - 1) == -2


def test_attention_refusals_and_sizes():
    L = dard.lib()
    def f(q=P, kc=P, ks=P, vc=P, vs=P, Pn=10, cap=64, state=P, conf=P, b=1, B=4, Hq=4, Hkv=2, dh=128, flags=0, out=P, ws=P,
          n=BIG):
        return L.dard_masked_attention_mx(q, kc, ks, vc, vs, Pn, None, cap, state, conf, b, B, Hq, Hkv, dh, 0.1, flags, out,
                                          ws, n, None)
    assert f(q=None) == -1 and f(state=None) == -1 and f(conf=None) == -1 and f(out=None) == -1 and f(vc=None) == -1
    assert f(flags=1 << 12) == -1 and f(flags=dard.F_C_BIDIR | dard.F_ORDER_L2R) == -1
    assert f(B=0) == -2 and f(B=257) == -2 and f(b=0) == -2 and f(Pn=-1) == -2 and f(Hq=5) == -2 and f(dh=96) == -2
    assert f(cap=48) == -2 and f(Pn=57) == -2 and f(Pn=2 ** 31 - 1) == -2 and f(B=40) == -2
    assert f(q=ctypes.c_void_p(0x1008)) == -1 and f(vs=ctypes.c_void_p(0x1004)) == -1
    need = L.dard_attention_mx_workspace_bytes(1, 4, 4, 2, 128, 20000)
    assert need > 0
    assert f(Pn=20000, cap=20032, n=need - 1) == -5 and f(Pn=20000, cap=20032, ws=None, n=0) == -5
    assert f(Pn=20000, cap=20032, ws=ctypes.c_void_p(0x1008)) == -1
    assert L.dard_attention_mx_workspace_bytes(1, 0, 4, 2, 128, 20) == 0
    assert L.dard_attention_mx_workspace_bytes(1, 4, 4, 2, 128, 2 ** 31 - 1) == 0


def test_binding_refusals():
    """What the binding refuses before it calls the library (CPU tensors reach no kernel)."""
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)   # noqa: E731
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError, match="device"):
        dard.dard_quantize_mx(x, dard.MX_FP8, u8(4, 64), u8(4, 2))
    for what, codes, scales in (("bytes", u8(4, 32), u8(4, 2)), ("bytes", u8(4, 64), u8(4, 3)), ("uint8", x, u8(4, 2))):
        with pytest.raises(ValueError, match=what):
            dard._mx_check(4, 64, dard.MX_FP8, codes, scales)
    with pytest.raises(ValueError, match="format"):
        dard._mx_check(4, 64, 2, u8(4, 64), u8(4, 2))
    with pytest.raises(ValueError, match="blocks"):
        dard._mx_check(4, 48, 0, u8(4, 48), u8(4, 1))
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        dard._mx_dt(x.half(), "x")
    with pytest.raises(ValueError, match="h must be float32"):
        dard.dard_resid_norm_mx(x.bfloat16(), x[0], 0.0, dard.MX_FP8, u8(4, 64), u8(4, 2))
    with pytest.raises(ValueError, match="gain"):
        dard.dard_resid_norm_mx(x, x[0, :32], 0.0, dard.MX_FP8, u8(4, 64), u8(4, 2))
    with pytest.raises(ValueError, match="packed"):
        dard.dard_linear_mx(dard.MX_FP8, u8(4, 64), u8(4, 2), u8(100), torch.zeros(4, 64))
    cache = [u8(2, 3, 64, 32), u8(2, 3, 64, 2), u8(2, 3, 8, 16, 8, 2), u8(2, 3, 8, 2, 8)]
    k = torch.zeros(2, 5, 3, 64)
    with pytest.raises(ValueError, match="one type"):
        dard.dard_kv_write_mx(k, k.bfloat16(), cache, 0)
    with pytest.raises(ValueError, match="vs must be"):
        dard.dard_kv_write_mx(k, k, cache[:3] + [u8(2, 3, 8, 8, 2)], 0)
    with pytest.raises(ValueError, match="kc must be"):
        dard.dard_kv_write_mx(k[:1], k[:1], cache, 0)
    q = torch.zeros(2, 4, 6, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="state and conf"):
        dard.dard_masked_attention_mx(q, cache, 0, u8(2, 4), torch.zeros(2, 4), 0.1, 0, q)
    with pytest.raises(ValueError, match="bfloat16"):
        dard.dard_masked_attention_mx(q.float(), cache, 0, u8(2, 2), torch.zeros(2, 2), 0.1, 0, q)
    with pytest.raises(ValueError, match="prefix"):
        dard._mx_prefix(torch.zeros(2, dtype=torch.int64), 2)


# ------------------------------------------------------------------ the plain forms themselves
def test_reference_formats():
    assert R.F8[0x7E] == 448 and R.F8[1] == 2.0 ** -9 and R.F8[8] == 2.0 ** -6 and np.isnan(R.F8[0x7F])
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(R.F8, t, equal_nan=True)
    x = np.zeros((1, 32))
    assert R.quantize(x, R.FP4)[1][0, 0] == 0
    x[0, :6] = 7.0, 5.0, 2.5, -1.75, 0.25, 0.75   # scale 1: saturation, ties to the even code
    c, s = R.quantize(x, R.FP4)
    assert s[0, 0] == 127
    assert list(R.values(c, s, R.FP4)[0, :6]) == [6.0, 4.0, 2.0, -2.0, 0.0, 1.0]
    x[0, 0] = 500.0                                 # scale 2^0 for E4M3 (256 <= 500 < 512): saturates at 448
    c, s = R.quantize(x, R.FP8)
    assert s[0, 0] == 127 and R.values(c, s, R.FP8)[0, 0] == 448


@pytest.mark.parametrize("fmt", [R.FP8, R.FP4])
def test_reference_quantize_is_nearest(fmt):
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 64)) * 10
    c, s = R.quantize(x, fmt)
    v = R.values(c, s, fmt)
    step = np.repeat(np.ldexp(1.0, s.astype(int) - 127), 32, -1)
    grid = np.unique((R.F8 if fmt == R.FP8 else R.F4)[~np.isnan(R.F8 if fmt == R.FP8 else R.F4)])
    best = np.abs(x[..., None] / step[..., None] - grid).min(-1) * step
    assert np.allclose(np.abs(x - v), best, rtol=0, atol=1e-12)
    assert np.array_equal(R.unpack(R.pack(c, fmt), fmt), c)


def test_reference_cache_layout():
    rng = np.random.default_rng(1)
    codes, scales = rng.integers(0, 256, (2, 3, 24, 32), dtype=np.uint8), rng.integers(0, 256, (2, 3, 24, 2), dtype=np.uint8)
    vc, vs = R.grouped(codes, scales)
    assert vc.shape == (2, 3, 3, 16, 8, 2) and vs.shape == (2, 3, 3, 2, 8)
    for s, h, key, byte in ((0, 0, 0, 0), (1, 2, 13, 31), (0, 1, 23, 6)):
        assert vc[s, h, key // 8, byte // 2, key % 8, byte % 2] == codes[s, h, key, byte]
        assert vs[s, h, key // 8, byte // 16, key % 8] == scales[s, h, key, byte // 16]
    c, sc = R.rows_of_cache(vc, vs)
    assert np.array_equal(c, codes) and np.array_equal(sc, scales)


def test_size_limits():
    L = dard.lib()
    assert L.dard_packed_mx_bytes(1, (1 << 20) + 32) == 0 and L.dard_packed_mx_bytes(1, 1 << 20) > 0
    assert L.dard_linear_mx(0, P, P, 1 << 30, 32, P, 1 << 20, 0, P, None, 0, None) == -2
    assert L.dard_linear_mx(0, P, P, 2 ** 31 - 1, 32, P, 1, 0, P, None, 0, None) == -2
    assert L.dard_resid_norm_mx(P, 0, None, 0, P, 1e-5, 1 << 24, 32, 0, P, P, None) == -2
    assert L.dard_quantize_mx(0, P, 32, 1 << 30, 32, 0, P, P, None) == -2
    f = lambda b, scale: L.dard_masked_attention_mx(   # noqa: E731
        P, P, P, P, P, 10, None, 64, P, P, b, 1, 4, 4, 128, scale, 0, P, P, BIG, None)
    assert f(1 << 22, 0.1) == -2   # 2^24 workgroups
    for scale in (0.0, -0.1, float("inf"), float("nan")):
        assert f(1, scale) == -1


def test_attention_scale_limit():
    """scale * log2(e), which the kernel takes, has to be a float32 too."""
    L = dard.lib()
    f = lambda scale: L.dard_masked_attention_mx(   # noqa: E731
        P, P, P, P, P, 10, None, 64, P, P, 1, 1, 4, 4, 128, scale, 0, P, None, 0, None)
    for scale in (2.0 ** 127, 3.4e38):
        assert f(scale) == -1 and b"scale" in L.dard_last_error()


def test_sizes_near_the_largest_int():
    """Sizes that rounding up would take past 2^31 - 1 are refused, not wrapped."""
    L = dard.lib()
    top = 2 ** 31 - 1
    for N in (top, top - 30):
        L.dard_packed_mx_bytes(0, 0)
        assert L.dard_packed_mx_bytes(N, 64) == 0 and b"2 GiB" in L.dard_last_error()
    assert L.dard_packed_mx_bytes(64, top - 31) == 0 and b"2^20" in L.dard_last_error()
