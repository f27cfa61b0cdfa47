// Product with MXFP4 weights: Y[m][n] = sum_k x[m][k] w[n][k], x in MXFP8 or
// MXFP4, on the scaled matrix instruction v_mfma_scale_f32_32x32x64_f8f6f4,
// which multiplies the elements, applies both blocks' scales and accumulates in
// fp32.  Its operands, for lane l (row l % 32, eta = l / 32) of a 64-k step:
//   E2M1: the 16 bytes of the block k = 32 eta .. 32 eta + 31;
//   E4M3: the 16 bytes from k = 16 eta and the 16 from k = 32 + 16 eta;
//   scale: the byte of the block 32 eta .. 32 eta + 31, taken from one of the
//   four bytes of a register: a register serves 256 k (a "unit").
// Inside the instruction the products of a group of eight consecutive k are
// aligned to the largest and cut 13 bits below its leading one (measured: a
// power of two 2^-14 of it no longer counts, neither does anything past 23 bits
// below the sum it is added to).
#include "launch.h"
#include "mx.h"

namespace dard {

namespace {

// One 64-k step; J picks the scale byte of both operands.
template <int F, int J>
__device__ __forceinline__ floatx16 mfma_mx(intx8 x, intx8 w, floatx16 c, uint32_t sx, uint32_t sw) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, w, c, Mx<F>::kMfma, Mx<DARD_MX_FP4>::kMfma, J, (int)sx, J,
                                                           (int)sw);
}

__device__ __forceinline__ intx8 ops(uint4 a, uint4 b) {
    return intx8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// X operand of step j of unit u for a row of K values (xr: its codes), zero past K.
template <int F> __device__ __forceinline__ intx8 ld_x(const uint8_t* xr, int u, int j, int eta, int K) {
    const uint4 zero = make_uint4(0, 0, 0, 0);
    const int k0 = 256 * u + 64 * j;
    if constexpr (F == DARD_MX_FP8) {
        const int ka = k0 + 16 * eta, kb = ka + 32;
        const uint4 a = ka < K ? *reinterpret_cast<const uint4*>(xr + ka) : zero;
        const uint4 b = kb < K ? *reinterpret_cast<const uint4*>(xr + kb) : zero;
        return ops(a, b);
    } else {
        const int ka = k0 + 32 * eta;
        return ops(ka < K ? *reinterpret_cast<const uint4*>(xr + ka / 2) : zero, zero);
    }
}

// Scales of a row's unit u: byte j = block 8 u + 2 j + eta (KB blocks a row, zero past them).
__device__ __forceinline__ uint32_t ld_xs(const uint8_t* xs, int u, int eta, int KB) {
    uint32_t w = 0;
    if (8 * u + 8 <= KB) {
        const Bytes8 b = *reinterpret_cast<const Bytes8*>(xs + 8 * u);
        w = __builtin_amdgcn_perm(b.y, b.x, eta ? 0x07050301u : 0x06040200u);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int kb = 8 * u + 2 * j + eta;
            if (kb < KB) w |= (uint32_t)xs[kb] << (8 * j);
        }
    }
    return w;
}

struct LinArgs {
    const uint8_t* xc; const uint8_t* xs; const uint8_t* wc; const uint32_t* ws;
    int M, K, N, KBp, nblk;
    int bf16_out;
    void* y;
    float* part;   // [split][M][N] when the K range is split over workgroups
};

__device__ __forceinline__ void st_y(const LinArgs& a, int m, int n, float v) {
    const size_t o = (size_t)m * a.N + n;
    if (a.bf16_out) reinterpret_cast<bf16_t*>(a.y)[o] = f2bf(v);
    else reinterpret_cast<float*>(a.y)[o] = v;
}

// A workgroup makes a tile of 32 MT rows x 32 NB columns; its NW waves split
// the K units and merge their sums through LDS.  Operands go from memory
// straight to registers.
template <int F, int MT, int NB, int NW>
__global__ __launch_bounds__(64 * NW) void linear_mx_kernel(LinArgs a) {
    __shared__ floatx4 red[NW][MT * NB * 4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, eta = lane >> 5;
    const int nb0 = blockIdx.x * NB, m0 = blockIdx.y * 32 * MT;
    const int units = a.KBp / 8, parts = NW * gridDim.z, pi = blockIdx.z * NW + wave;
    const int u0 = (int)((int64_t)units * pi / parts), u1 = (int)((int64_t)units * (pi + 1) / parts);
    const int KB = a.K / 32;
    floatx16 acc[MT][NB];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = floatx16{};
    const uint8_t* xr[MT];
    const uint8_t* xsr[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const size_t m = min(m0 + 32 * i + r, a.M - 1);
        xr[i] = a.xc + m * (F == DARD_MX_FP8 ? a.K : a.K / 2);
        xsr[i] = a.xs + m * KB;
    }
    for (int u = u0; u < u1; ++u) {
        uint32_t sx[MT], sw[NB];
        uint4 w[NB][4];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const size_t blk = min(nb0 + j, a.nblk - 1);
            sw[j] = a.ws[(blk * units + u) * 64 + lane];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                w[j][q] = reinterpret_cast<const uint4*>(a.wc)[(blk * a.KBp + 8 * u + 2 * q + eta) * 32 + r];
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) sx[i] = ld_xs(xsr[i], u, eta, KB);
        intx8 x[MT][4];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) x[i][q] = ld_x<F>(xr[i], u, q, eta, a.K);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const uint4 z = make_uint4(0, 0, 0, 0);
                acc[i][j] = mfma_mx<F, 0>(x[i][0], ops(w[j][0], z), acc[i][j], sx[i], sw[j]);
                acc[i][j] = mfma_mx<F, 1>(x[i][1], ops(w[j][1], z), acc[i][j], sx[i], sw[j]);
                acc[i][j] = mfma_mx<F, 2>(x[i][2], ops(w[j][2], z), acc[i][j], sx[i], sw[j]);
                acc[i][j] = mfma_mx<F, 3>(x[i][3], ops(w[j][3], z), acc[i][j], sx[i], sw[j]);
            }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                red[wave][(i * NB + j) * 4 + q][lane] =
                    floatx4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    __syncthreads();
    // element 4 q + c of a tile: row 8 q + 4 eta + c, column lane % 32
    for (int t = wave; t < MT * NB * 4; t += NW) {
        floatx4 v = red[0][t][lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) v += red[w][t][lane];
        const int q = t & 3, tile = t >> 2;
        const int m = m0 + 32 * (tile / NB) + 8 * q + 4 * eta, n = (nb0 + tile % NB) * 32 + r;
        if (n >= a.N) continue;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (m + c >= a.M) continue;
            if (gridDim.z > 1) a.part[((size_t)blockIdx.z * a.M + m + c) * a.N + n] = v[c];
            else st_y(a, m + c, n, v[c]);
        }
    }
}

// Sum of the K splits' partials, in split order.
__global__ __launch_bounds__(256) void linear_mx_sum_kernel(LinArgs a, int nsplit, int64_t total) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= total) return;
    float v = a.part[i];
    for (int s = 1; s < nsplit; ++s) v += a.part[s * total + i];
    if (a.bf16_out) reinterpret_cast<bf16_t*>(a.y)[i] = f2bf(v);
    else reinterpret_cast<float*>(a.y)[i] = v;
}

struct Plan {
    int nt, mt, split;
};

Plan plan_of(int, int M, int N, int K) {
    Plan p;
    p.nt = (N + 63) / 64;
    p.mt = (M + 63) / 64;
    const int units = (K / 32 + 7) / 8;
    p.split = 1;
    while (p.nt * p.mt * p.split < 256 && units / (p.split * 2 * 4) >= 1 && p.split < 8) p.split *= 2;
    return p;
}

template <int F> void run(const LinArgs& a, const Plan& p, hipStream_t s) {
    launch(linear_mx_kernel<F, 2, 2, 4>, dim3(p.nt, p.mt, p.split), dim3(256), 0, s, a);
}

}  // namespace

size_t linear_mx_partial_bytes(int format, int M, int N, int K) {
    const Plan p = plan_of(format, M, N, K);
    return p.split > 1 ? (size_t)p.split * M * N * 4 : 0;
}

hipError_t launch_linear_mx(int format, const uint8_t* xc, const uint8_t* xs, int M, int K, const void* Wp, int N,
                            int out_dtype, void* y, float* part, hipStream_t s) {
    const MxPacked w = mx_packed(N, K);
    const Plan p = plan_of(format, M, N, K);
    LinArgs a{};
    a.xc = xc; a.xs = xs; a.wc = (const uint8_t*)Wp; a.ws = (const uint32_t*)((const char*)Wp + w.scales);
    a.M = M; a.K = K; a.N = N; a.KBp = w.KBp; a.nblk = w.nblk;
    a.bf16_out = out_dtype == DARD_DTYPE_BF16;
    a.y = y; a.part = part;
    if (format == DARD_MX_FP8) run<DARD_MX_FP8>(a, p, s);
    else run<DARD_MX_FP4>(a, p, s);
    if (p.split > 1) {
        const int64_t total = (int64_t)M * N;
        launch(linear_mx_sum_kernel, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, s, a, p.split, total);
    }
    return hipGetLastError();
}

}  // namespace dard
