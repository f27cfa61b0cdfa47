// Microscaled (MX) formats: quantisation of rows, its inverse, the residual
// norm with MX output, the packed weight image of the MX product, and the
// MXFP4 KV cache's writer and reader.  All of these move bytes: each thread
// takes 8 consecutive values, the four lanes of a quad share a block of 32.
#include "launch.h"
#include "mx.h"

namespace dard {

namespace {

// Codes of 8 values to row-major storage (chunk c of 8 values).
template <int F> __device__ __forceinline__ void st_codes(uint8_t* codes, size_t c, uint2 w) {
    if constexpr (F == DARD_MX_FP8)
        *reinterpret_cast<uint2*>(codes + 8 * c) = w;
    else
        *reinterpret_cast<uint32_t*>(codes + 4 * c) = w.x;
}

// Eight values of a quad's block to codes and the block's scale byte.  The
// product with a power of two is exact unless it underflows, and then the
// value rounds to zero in either type.
template <int F> __device__ __forceinline__ uint2 quantize8(const float (&v)[8], uint32_t& scale) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(v[i]) & 0x7FFFFFFFu;
        top = a > top ? a : top;
    }
    scale = mx_scale<F>(quad_max(top) >> 23);
    const float inv = scale == 255u ? 0.f : __uint_as_float((254u - scale) << 23);
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = scale == 255u ? 0.f : v[i] * inv;
    return mx_encode8<F>(t);
}

// At the rate of a copy: 8192 x 3584 bf16 from memory to MXFP4 in 16.1 us, 4.6 TB/s (to MXFP8 19.5 us, float32 to
// MXFP4 23.7, 5.6 TB/s); four chunks a thread in flight gain nothing.  Right behind a product that left its
// output dirty in the caches the same call takes 24 us.
template <typename T, int F>
__global__ __launch_bounds__(256) void quantize_mx_kernel(const T* __restrict__ x, int64_t ld, uint32_t nchunk, uint32_t cpr,
                                                          uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    // (a quad's chunks are of one row and inside or outside together: cpr % 4 == 0)
    const uint32_t c = blockIdx.x * 256u + threadIdx.x;
    if (c >= nchunk) return;
    const uint32_t row = c / cpr;
    float v[8];
    ld_8(x + row * ld + 8 * (c - row * cpr), v);
    uint32_t scale;
    const uint2 w = quantize8<F>(v, scale);
    st_codes<F>(codes, c, w);
    if ((c & 3) == 0) scales[c >> 2] = (uint8_t)scale;
}

// Bound by its bytes: 8192 x 3584 MXFP8 to bf16 in 18.5 us, 4.8 TB/s (MXFP4 18.7, 4.0 TB/s), to float32 29.8 us, 5.0
// TB/s (MXFP4 29.9, 4.4).
template <typename T, int F>
__global__ __launch_bounds__(256) void dequantize_mx_kernel(const uint8_t* __restrict__ codes,
                                                            const uint8_t* __restrict__ scales, uint32_t nchunk,
                                                            uint32_t cpr, T* __restrict__ x, int64_t ld) {
    const size_t c = blockIdx.x * 256u + threadIdx.x;
    if (c >= nchunk) return;
    const uint32_t row = (uint32_t)c / cpr;
    T* out = x + row * ld + 8 * (c - (size_t)row * cpr);
    const uint32_t sb = scales[c >> 2];
    // scale 0 is 2^-127 (a subnormal float), 255 NaN
    const float s = sb == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(sb ? sb << 23 : 0x00400000u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t code = F == DARD_MX_FP8 ? (uint32_t)codes[8 * c + i] : (uint32_t)codes[4 * c + i / 2] >> (4 * (i & 1));
        St<T>::st(out + i, mx_value<F>(code) * s);
    }
}

// h += delta (rounded once to float32, stored), y = h gain / sqrt(mean(h^2) + eps),
// y in MX.  One workgroup per row, the row in registers.  The norm is evaluated
// in 64 bits up to the element's rounding (the memory traffic hides it): an
// 8-bit step is so coarse that a last bit of a float32 sum, which depends on
// how a row is split, would now and then move a value by a whole step.
// Bound by its bytes: 8192 x 3584 with a bf16 delta to MXFP8 in 63.9 us, 5.07 TB/s, a
// copy's rate; 64 x 4096 in 4.6 us, a launch and two trips to memory.
template <int NV, typename D, typename G, int F>
__global__ __launch_bounds__(256) void resid_norm_mx_kernel(float* __restrict__ h, const D* __restrict__ delta,
                                                            const G* __restrict__ gain, float eps, int d,
                                                            uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    __shared__ double red[4];
    const int t = threadIdx.x, nt = blockDim.x, cpr = d / 8;
    const size_t row = blockIdx.x;
    float* hr = h + row * d;
    float v[NV][8];
    double ss = 0.0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = t + i * nt;
        if (c >= cpr) continue;
        ld_8(hr + 8 * c, v[i]);
        if (delta) {
            float a[8];
            ld_8(delta + row * d + 8 * c, a);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] += a[e];
            floatx4 lo, hi;
#pragma unroll
            for (int e = 0; e < 4; ++e) { lo[e] = v[i][e]; hi[e] = v[i][4 + e]; }
            st_f4(hr + 8 * c, lo);
            st_f4(hr + 8 * c + 4, hi);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fma((double)v[i][e], (double)v[i][e], ss);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o, 64);
    if ((t & 63) == 0) red[t >> 6] = ss;
    __syncthreads();
    ss = 0.0;
    for (int i = 0; i < nt / 64; ++i) ss += red[i];
    const double rs = 1.0 / sqrt(ss / (double)d + (double)eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = t + i * nt;
        if (c >= cpr) continue;
        float g[8];
        ld_8(gain + 8 * c, g);
        double y[8];
        uint32_t top = 0;   // upper words of the magnitudes: they hold the exponent
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            y[e] = (double)v[i][e] * rs * (double)g[e];
            const uint32_t hi = (uint32_t)__double2hiint(y[e]) & 0x7FFFFFFFu;
            top = hi > top ? hi : top;
        }
        const int E = (int)(quad_max(top) >> 20);
        int code = E - 1023 + 127 - Mx<F>::kEmax;
        code = code < 0 ? 0 : (code > 254 ? 254 : code);
        if (E == 0x7FF) code = 255;
        const double inv = __hiloint2double((1023 + 127 - code) << 20, 0);
        float q[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // to kMant fractional digits below the leading one (the smallest exponent's
            // step below kEmin): adding and taking away 1.5 * 2^(52 - digits) rounds once,
            // to nearest even (and a small negative value keeps its sign)
            const double x = code == 255 ? 0.0 : y[e] * inv;
            int ex = (int)(((uint32_t)__double2hiint(x) >> 20) & 0x7FFu);
            ex = ex < 1023 + Mx<F>::kEmin ? 1023 + Mx<F>::kEmin : ex;
            const double magic = __hiloint2double(((ex + 52 - Mx<F>::kMant) << 20) | 0x80000, 0);
            q[e] = copysignf((float)((x + magic) - magic), __int_as_float(__double2hiint(x)));
        }
        const uint2 w = mx_encode8<F>(q);
        const size_t cc = row * cpr + c;
        st_codes<F>(codes, cc, w);
        if ((c & 3) == 0) scales[cc >> 2] = (uint8_t)code;
    }
}

// Packed weights of the MX product (see mx_linear.hip): one thread per 16-byte
// block of 32 codes, or per dword of four scales.
__global__ __launch_bounds__(256) void pack_mx_kernel(const uint4* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                      int N, int KB, int KBp, int64_t ncode, int64_t nscale,
                                                      uint4* __restrict__ wc, uint32_t* __restrict__ ws) {
    int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < ncode) {
        const int r = (int)(i & 31);
        const int64_t j = i >> 5;
        const int kb = (int)(j % KBp);
        const int64_t n = (j / KBp) * 32 + r;
        wc[i] = n < N && kb < KB ? codes[n * KB + kb] : make_uint4(0, 0, 0, 0);
        return;
    }
    i -= ncode;
    if (i >= nscale) return;
    const int lane = (int)(i & 63), r = lane & 31, eta = lane >> 5;
    const int64_t j = i >> 6;
    const int u = (int)(j % (KBp / 8));
    const int64_t n = (j / (KBp / 8)) * 32 + r;
    uint32_t w = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int kb = 8 * u + 2 * q + eta;
        if (n < N && kb < KB) w |= (uint32_t)scales[n * KB + kb] << (8 * q);
    }
    ws[i] = w;
}

// Position of a sequence's first new key.
__device__ __forceinline__ int kv_first(const int32_t* prefix, int pos, int s) {
    if (!prefix) return pos;
    const int p = prefix[s];
    return p < 0 ? 0 : (p > pos ? pos : p);
}

// Chunk c of 8 dims of KV head h of new key t of sequence s, the i-th of a call (32-bit divisions: a call has
// under 2^31 of them).
struct KvItem {
    int c, h, t, s;
};
__device__ __forceinline__ KvItem kv_item(const MxKvArgs& a, uint32_t i) {
    const uint32_t sh = a.dh == 128 ? 4 : 3, key = i >> sh, st = key / (uint32_t)a.Hkv, s = st / (uint32_t)a.n;
    return {(int)(i & ((1u << sh) - 1)), (int)(key - st * a.Hkv), (int)(st - s * a.n), (int)s};
}

// One thread per 8 dims of one key of K (blockIdx.y = 0) or V (1), a key's dims and heads next to each other.  Bound
// by bytes and, for V, by accesses: a lane's codes are two bytes here and two 16 bytes on, the other keys of the group
// lie between.  8192 float32 keys of 4 heads x 128 take 9.1 us (38 MB), reading them back as bf16 7.2 us
// (21 MB); 64 keys of 32 heads 3.0 us each.
template <typename T>
__global__ __launch_bounds__(256) void kv_write_mx_kernel(MxKvArgs a, const T* __restrict__ k, const T* __restrict__ v) {
    const KvItem item = kv_item(a, blockIdx.x * 256u + threadIdx.x);
    if (item.s >= a.b) return;
    const int cpk = a.dh / 8, c = item.c, h = item.h, s = item.s, t = item.t;
    const int64_t st = (int64_t)s * a.n + t;
    const bool is_v = blockIdx.y;
    const T* src = (is_v ? v : k) + st * a.ld + (int64_t)h * a.dh + 8 * c;
    const size_t key = (size_t)kv_first(a.prefix, a.pos, s) + t, roitem = ((size_t)s * a.Hkv + h) * a.cap;
    float x[8];
    ld_8(src, x);
    uint32_t scale;
    const uint32_t w = quantize8<DARD_MX_FP4>(x, scale).x;
    if (!is_v) {
        reinterpret_cast<uint32_t*>(a.kc)[(roitem + key) * cpk + c] = w;
        if ((c & 3) == 0) a.ks[(roitem + key) * (a.dh / 32) + (c >> 2)] = (uint8_t)scale;
    } else {
        const size_t grp = (roitem + key) >> 3;
        uint16_t* dst = reinterpret_cast<uint16_t*>(a.vc) + (grp * (a.dh / 4) + 2 * c) * 8 + (key & 7);
        dst[0] = (uint16_t)w;
        dst[8] = (uint16_t)(w >> 16);
        if ((c & 3) == 0) a.vs[(grp * (a.dh / 32) + (c >> 2)) * 8 + (key & 7)] = (uint8_t)scale;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void kv_read_mx_kernel(MxKvArgs a, T* __restrict__ k, T* __restrict__ v) {
    const KvItem item = kv_item(a, blockIdx.x * 256u + threadIdx.x);
    if (item.s >= a.b) return;
    const int cpk = a.dh / 8, c = item.c, h = item.h, s = item.s, t = item.t;
    const int64_t st = (int64_t)s * a.n + t;
    const bool is_v = blockIdx.y;
    T* dst = (is_v ? v : k) + st * a.ld + (int64_t)h * a.dh + 8 * c;
    const size_t key = (size_t)kv_first(a.prefix, a.pos, s) + t, roitem = ((size_t)s * a.Hkv + h) * a.cap;
    uint32_t w, sb;
    if (!is_v) {
        w = reinterpret_cast<const uint32_t*>(a.kc)[(roitem + key) * cpk + c];
        sb = a.ks[(roitem + key) * (a.dh / 32) + (c >> 2)];
    } else {
        const size_t grp = (roitem + key) >> 3;
        const uint16_t* src = reinterpret_cast<const uint16_t*>(a.vc) + (grp * (a.dh / 4) + 2 * c) * 8 + (key & 7);
        w = (uint32_t)src[0] | ((uint32_t)src[8] << 16);
        sb = a.vs[(grp * (a.dh / 32) + (c >> 2)) * 8 + (key & 7)];
    }
    // E2M1 times a power of two is exact in bf16, and in float32
    const float f = mx_scale_f(sb);
    const uint32_t p[4] = {fp4x2_to_bf16x2<0>(w, f), fp4x2_to_bf16x2<1>(w, f), fp4x2_to_bf16x2<2>(w, f),
                           fp4x2_to_bf16x2<3>(w, f)};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        St<T>::st(dst + 2 * j, __uint_as_float(p[j] << 16));
        St<T>::st(dst + 2 * j + 1, __uint_as_float(p[j] & 0xFFFF0000u));
    }
}

unsigned blocks256(int64_t n) { return (unsigned)((n + 255) / 256); }

template <int NV, typename D, typename G, int F>
void run_norm(float* h, const void* delta, const void* gain, float eps, int rows, int d, uint8_t* codes, uint8_t* scales,
              int nt, hipStream_t s) {
    launch(resid_norm_mx_kernel<NV, D, G, F>, dim3(rows), dim3(nt), 0, s, h, (const D*)delta, (const G*)gain, eps, d,
           codes, scales);
}

template <typename D, typename G, int F>
void run_norm_nv(float* h, const void* delta, const void* gain, float eps, int rows, int d, uint8_t* codes,
                 uint8_t* scales, hipStream_t s) {
    const int cpr = d / 8;
    const int nt = cpr >= 256 ? 256 : (cpr + 63) / 64 * 64;
    switch ((cpr + nt - 1) / nt) {
        case 1: run_norm<1, D, G, F>(h, delta, gain, eps, rows, d, codes, scales, nt, s); break;
        case 2: run_norm<2, D, G, F>(h, delta, gain, eps, rows, d, codes, scales, nt, s); break;
        case 3: run_norm<3, D, G, F>(h, delta, gain, eps, rows, d, codes, scales, nt, s); break;
        default: run_norm<4, D, G, F>(h, delta, gain, eps, rows, d, codes, scales, nt, s); break;
    }
}

template <typename D, typename G>
void run_norm_f(int format, float* h, const void* delta, const void* gain, float eps, int rows, int d, uint8_t* codes,
                uint8_t* scales, hipStream_t s) {
    if (format == DARD_MX_FP8)
        run_norm_nv<D, G, DARD_MX_FP8>(h, delta, gain, eps, rows, d, codes, scales, s);
    else
        run_norm_nv<D, G, DARD_MX_FP4>(h, delta, gain, eps, rows, d, codes, scales, s);
}

template <typename T, int F>
void run_quantize(const void* x, int64_t ld, int64_t n, int K, uint8_t* codes, uint8_t* scales, hipStream_t s) {
    launch(quantize_mx_kernel<T, F>, dim3(blocks256(n)), dim3(256), 0, s, (const T*)x, ld, (uint32_t)n, (uint32_t)(K / 8), codes,
           scales);
}

template <typename T, int F>
void run_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t n, int K, void* x, int64_t ld, hipStream_t s) {
    launch(dequantize_mx_kernel<T, F>, dim3(blocks256(n)), dim3(256), 0, s, codes, scales, (uint32_t)n, (uint32_t)(K / 8), (T*)x,
           ld);
}

}  // namespace

hipError_t launch_quantize_mx(int dtype, const void* x, int64_t ld, int64_t rows, int K, int format, uint8_t* codes,
                              uint8_t* scales, hipStream_t s) {
    const int64_t n = rows * (K / 8);
    const bool b = dtype == DARD_DTYPE_BF16, f8 = format == DARD_MX_FP8;
    if (b && f8) run_quantize<bf16_t, DARD_MX_FP8>(x, ld, n, K, codes, scales, s);
    else if (b) run_quantize<bf16_t, DARD_MX_FP4>(x, ld, n, K, codes, scales, s);
    else if (f8) run_quantize<float, DARD_MX_FP8>(x, ld, n, K, codes, scales, s);
    else run_quantize<float, DARD_MX_FP4>(x, ld, n, K, codes, scales, s);
    return hipGetLastError();
}

hipError_t launch_dequantize_mx(int format, const uint8_t* codes, const uint8_t* scales, int64_t rows, int K, int dtype,
                                void* x, int64_t ld, hipStream_t s) {
    const int64_t n = rows * (K / 8);
    const bool b = dtype == DARD_DTYPE_BF16, f8 = format == DARD_MX_FP8;
    if (b && f8) run_dequantize<bf16_t, DARD_MX_FP8>(codes, scales, n, K, x, ld, s);
    else if (b) run_dequantize<bf16_t, DARD_MX_FP4>(codes, scales, n, K, x, ld, s);
    else if (f8) run_dequantize<float, DARD_MX_FP8>(codes, scales, n, K, x, ld, s);
    else run_dequantize<float, DARD_MX_FP4>(codes, scales, n, K, x, ld, s);
    return hipGetLastError();
}

hipError_t launch_resid_norm_mx(float* h, int delta_dtype, const void* delta, int gain_dtype, const void* gain, float eps,
                                int rows, int d, int format, uint8_t* codes, uint8_t* scales, hipStream_t s) {
    const bool db = delta_dtype == DARD_DTYPE_BF16, gb = gain_dtype == DARD_DTYPE_BF16;
    if (db && gb) run_norm_f<bf16_t, bf16_t>(format, h, delta, gain, eps, rows, d, codes, scales, s);
    else if (db) run_norm_f<bf16_t, float>(format, h, delta, gain, eps, rows, d, codes, scales, s);
    else if (gb) run_norm_f<float, bf16_t>(format, h, delta, gain, eps, rows, d, codes, scales, s);
    else run_norm_f<float, float>(format, h, delta, gain, eps, rows, d, codes, scales, s);
    return hipGetLastError();
}

hipError_t launch_pack_mx(const void* codes, const uint8_t* scales, int N, int K, void* Wp, hipStream_t s) {
    const MxPacked p = mx_packed(N, K);
    const int64_t ncode = (int64_t)p.nblk * p.KBp * 32, nscale = (int64_t)p.nblk * (p.KBp / 8) * 64;
    launch(pack_mx_kernel, dim3(blocks256(ncode + nscale)), dim3(256), 0, s, (const uint4*)codes, scales, N, K / 32, p.KBp,
           ncode, nscale, (uint4*)Wp, (uint32_t*)((char*)Wp + p.scales));
    return hipGetLastError();
}

hipError_t launch_kv_write_mx(int dtype, const MxKvArgs& a, const void* k, const void* v, hipStream_t s) {
    const int64_t total = (int64_t)a.b * a.n * a.Hkv * (a.dh / 8);
    const dim3 g(blocks256(total), 2);
    if (dtype == DARD_DTYPE_BF16)
        launch(kv_write_mx_kernel<bf16_t>, g, dim3(256), 0, s, a, (const bf16_t*)k, (const bf16_t*)v);
    else
        launch(kv_write_mx_kernel<float>, g, dim3(256), 0, s, a, (const float*)k, (const float*)v);
    return hipGetLastError();
}

hipError_t launch_kv_read_mx(int dtype, const MxKvArgs& a, void* k, void* v, hipStream_t s) {
    const int64_t total = (int64_t)a.b * a.n * a.Hkv * (a.dh / 8);
    const dim3 g(blocks256(total), 2);
    if (dtype == DARD_DTYPE_BF16)
        launch(kv_read_mx_kernel<bf16_t>, g, dim3(256), 0, s, a, (bf16_t*)k, (bf16_t*)v);
    else
        launch(kv_read_mx_kernel<float>, g, dim3(256), 0, s, a, (float*)k, (float*)v);
    return hipGetLastError();
}

}  // namespace dard
