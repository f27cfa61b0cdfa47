// Product with MXFP4 weights: Y[m][n] = sum_k x[m][k] w[n][k], x in MXFP8 or
// MXFP4, on the scaled matrix instruction v_mfma_scale_f32_32x32x64_f8f6f4,
// which multiplies the elements, applies both blocks' scales and accumulates in
// fp32 (fp32 results of MXFP8 rows: on the bf16 one, see XFrag).  Its operands, for lane l (row l % 32, eta = l / 32) of a 64-k step:
//   E2M1: the 16 bytes of the block k = 32 eta .. 32 eta + 31;
//   E4M3: the 16 bytes from k = 16 eta and the 16 from k = 32 + 16 eta;
//   scale: the byte of the block 32 eta .. 32 eta + 31, taken from one of the
//   four bytes of a register: a register serves 256 k (a "unit").
// Inside the instruction the products of a group of eight consecutive k are
// aligned to the largest and cut 13 bits below its leading one (measured: a
// power of two 2^-14 of it no longer counts, neither does anything past 23 bits
// below the sum it is added to).
#include <cmath>
#include <type_traits>

#include "launch.h"
#include "mx.h"

namespace dard {

namespace {

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));   // (vector types for LDS reads: see mx_attention.hip)

// Operands of one 64-k step.  Exact (EX): the step runs on v_mfma_f32_32x32x16_bf16 instead,
// both operands widened to bf16 with their scales (exact: at most 4 significant bits), so that
// sums are float32's own.  That has half the rate, and takes x in the k order of E2M1:
// both 16-byte chunks from k = 32 eta on.
template <int F> struct XFrag {
    uintx4 c[F == DARD_MX_FP8 ? 2 : 1];
};

// Chunk of 16 code bytes, of a step's, that part P of a lane's operand is.
template <int F, bool EX> __device__ __forceinline__ int x_chunk(int eta, int p) {
    if constexpr (F == DARD_MX_FP4) return eta;
    else return EX ? 2 * eta + p : eta + 2 * p;
}

template <int F> __device__ __forceinline__ bf16x8 widen8(const XFrag<F>& x, int q, float f) {   // values 8 q .. 8 q + 7
    uint32_t r[4];
    if constexpr (F == DARD_MX_FP8) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t w = x.c[q / 2][2 * (q & 1) + i];
            r[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, f, false));
            r[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, f, true));
        }
    } else {
        const uint32_t w = x.c[0][q];
        r[0] = fp4x2_to_bf16x2<0>(w, f);
        r[1] = fp4x2_to_bf16x2<1>(w, f);
        r[2] = fp4x2_to_bf16x2<2>(w, f);
        r[3] = fp4x2_to_bf16x2<3>(w, f);
    }
    return __builtin_bit_cast(bf16x8, uintx4{r[0], r[1], r[2], r[3]});
}

// acc += one 64-k step of TI x TJ blocks; byte J of the scale words is the step's.
template <int F, int J, int TI, int TJ>
__device__ __forceinline__ void mm_scaled(const XFrag<F> (&x)[TI], const uintx4 (&w)[TJ], const uint32_t (&sx)[TI],
                                          const uint32_t (&sw)[TJ], floatx16 (&acc)[TI][TJ]) {
#pragma unroll
    for (int i = 0; i < TI; ++i) {
        const uintx4 lo = x[i].c[0], hi = F == DARD_MX_FP8 ? x[i].c[F == DARD_MX_FP8 ? 1 : 0] : uintx4{0, 0, 0, 0};
        const intx8 xv = {(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
            const intx8 wv = {(int)w[j][0], (int)w[j][1], (int)w[j][2], (int)w[j][3], 0, 0, 0, 0};
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(xv, wv, acc[i][j], Mx<F>::kMfma, Mx<DARD_MX_FP4>::kMfma,
                                                                       J, (int)sx[i], J, (int)sw[j]);
        }
    }
}

template <int F, bool EX, int J, int TI, int TJ>
__device__ __forceinline__ void mm_step(const XFrag<F> (&x)[TI], const uintx4 (&w)[TJ], const uint32_t (&sx)[TI],
                                        const uint32_t (&sw)[TJ], floatx16 (&acc)[TI][TJ]) {
    if constexpr (!EX) {
        mm_scaled<F, J, TI, TJ>(x, w, sx, sw, acc);
    } else {
        float fx[TI], fw[TJ];   // (the conversions read the exponent field alone)
#pragma unroll
        for (int i = 0; i < TI; ++i) fx[i] = __uint_as_float(J < 3 ? sx[i] << (23 - 8 * J) : sx[i] >> 1);
#pragma unroll
        for (int j = 0; j < TJ; ++j) fw[j] = __uint_as_float(J < 3 ? sw[j] << (23 - 8 * J) : sw[j] >> 1);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            bf16x8 wv[TJ];
#pragma unroll
            for (int j = 0; j < TJ; ++j) {
                XFrag<DARD_MX_FP4> t;
                t.c[0] = w[j];
                wv[j] = widen8<DARD_MX_FP4>(t, q, fw[j]);
            }
#pragma unroll
            for (int i = 0; i < TI; ++i) {
                const bf16x8 xv = widen8<F>(x[i], q, fx[i]);
#pragma unroll
                for (int j = 0; j < TJ; ++j) acc[i][j] = mfma32x32x16(xv, wv[j], acc[i][j]);
            }
        }
    }
}

// Scale dwords of a row of x: rows of scales need not be dword-aligned, so N + 1 aligned dwords from
// byte `at` on are read and shifted; blocks past K (another row's) give zero.  `first`: the first
// block of the N dwords, KB blocks a row.  Bytes eta, eta + 2, ... are the lane's steps.
template <int N>
__device__ __forceinline__ uint32_t x_scales(const uint32_t (&d)[N + 1], int at, int first, int KB, int eta) {
    uint32_t v[N];
#pragma unroll
    for (int q = 0; q < N; ++q) {
        v[q] = __builtin_amdgcn_alignbyte(d[q + 1], d[q], at & 3);
        const int n = KB - first - 4 * q;
        v[q] = n >= 4 ? v[q] : n <= 0 ? 0u : v[q] & ((1u << (8 * n)) - 1u);
    }
    if constexpr (N == 2) return __builtin_amdgcn_perm(v[1], v[0], eta ? 0x07050301u : 0x06040200u);
    else return __builtin_amdgcn_perm(0u, v[0], eta ? 0x0C0C0301u : 0x0C0C0200u);
}

struct LinArgs {
    const uint8_t* xc; const uint8_t* xs; const uint8_t* wc; const uint32_t* ws;
    int M, K, N, KBp, nblk;
    int bf16_out;
    void* y;
};

// Bit 4 of each byte from 240 on.  Scales that high could take operands past bf16's range (x: codes from 247
// on, w: from 253 on; quantised float32 never has them) where their products are in range: elements
// of a row or column of a wave that met one are made again on the scaled instruction.
__device__ __forceinline__ uint32_t high_scales(uint32_t s) {
    const uint32_t t = s & (s >> 1);
    return t & (t >> 2) & 0x10101010u;
}
template <int TI, int TJ> struct High {   // bits 4 + i of the bytes: the lane's row (column) of block i
    uint32_t x = 0, w = 0;
    __device__ __forceinline__ void add(const uint32_t (&sx)[TI], const uint32_t (&sw)[TJ]) {
#pragma unroll
        for (int i = 0; i < TI; ++i) x |= high_scales(sx[i]) << i;
#pragma unroll
        for (int j = 0; j < TJ; ++j) w |= high_scales(sw[j]) << j;
    }
};
// Block (i, j) of the blocks of a wave, its first row m and column n, units u0 to u1, straight from memory:
// put(v, value) for the elements v of the lane that are to be replaced.
template <int TI, int TJ, typename Put>
__device__ __forceinline__ void redo_scaled(const LinArgs& a, int m, int n, int i, int j, int u0, int u1, const High<TI, TJ>& high,
                                            Put&& put) {
    const uint64_t bx = __ballot((high.x & 0x10101010u << i) != 0), bw = __ballot((high.w & 0x10101010u << j) != 0);
    if ((bx | bw) == 0) return;
    const int lane = threadIdx.x & 63, lr = lane & 31, eta = lane >> 5, KB = a.K / 32, units = a.KBp / 8;
    const size_t row = m + lr, blk = min(n / 32, a.nblk - 1);
    const bool in = row < (size_t)a.M;
    floatx16 t[1][1] = {{floatx16{}}};
#pragma unroll 1
    for (int st = 4 * u0; st < 4 * u1; ++st) {
        XFrag<DARD_MX_FP8> x[1];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int k = 64 * st + 16 * x_chunk<DARD_MX_FP8, false>(eta, p);
            x[0].c[p] = in && k < a.K ? *reinterpret_cast<const uintx4*>(a.xc + row * a.K + k) : uintx4{};
        }
        const uint32_t sx[1] = {in && 2 * st + eta < KB ? (uint32_t)a.xs[row * KB + 2 * st + eta] : 0u};
        const uintx4 w[1] = {*reinterpret_cast<const uintx4*>(a.wc + blk * a.KBp * 512 + (size_t)st * 1024 + 16 * lane)};
        const uint32_t sw[1] = {a.ws[(blk * units + st / 4) * 64 + lane] >> (8 * (st % 4))};
        mm_scaled<DARD_MX_FP8, 0, 1, 1>(x, w, sx, sw, t);
    }
    const uint32_t rows = (uint32_t)(bx | bx >> 32), col = (uint32_t)(bw | bw >> 32) >> lr & 1u;
#pragma unroll
    for (int v = 0; v < 16; ++v)
        if (col | (rows >> (8 * (v / 4) + 4 * eta + v % 4) & 1u)) put(v, t[0][0][v]);
}

__device__ __forceinline__ void st_y(const LinArgs& a, int m, int n, float v) {
    const size_t o = (size_t)m * a.N + n;
    if (a.bf16_out) reinterpret_cast<bf16_t*>(a.y)[o] = f2bf(v);
    else reinterpret_cast<float*>(a.y)[o] = v;
}

// The first n (all from 4 or 8 on) of 4 floats, or of 8 floats as bf16, at an address that is
// only as aligned as its element.
__device__ __forceinline__ void st_4(float* p, floatx4 v, int n) {
    if (n >= 4) {
        st_f4(p, v);
        return;
    }
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (e < n) p[e] = v[e];
}
__device__ __forceinline__ void st_8(bf16_t* p, floatx4 lo, floatx4 hi, int n) {
    typedef __bf16 b8 __attribute__((ext_vector_type(8), aligned(2)));
    const b8 w = __builtin_convertvector(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), bf16x8);
    if (n >= 8) {
        *reinterpret_cast<b8*>(p) = w;
        return;
    }
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < n) p[e] = __builtin_bit_cast(bf16_t, (__bf16)w[e]);
}

template <int SIZE> __device__ __forceinline__ void copy_lds(__amdgpu_buffer_rsrc_t r, char* dst, int voff, int soff) {
#if __HIP_DEVICE_COMPILE__   // (the host pass does not know the builtin)
    typedef __attribute__((address_space(3))) void* lds_ptr;
    if constexpr (SIZE == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr)dst, 16, voff, soff, 0, 0);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr)dst, 4, voff, soff, 0, 0);
#endif
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void* p, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)(bytes < 0xFFFFFF00ll ? bytes : 0xFFFFFF00ll),
                                             0x00020000);
}
// A descriptor of the scales of rows m0.. of x: based at the dword of the first, ending with the
// dword of the last.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_xs(const LinArgs& a, int m0, int KB, int& low) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(a.xs + (size_t)m0 * KB);
    low = (int)(p & 3);
    return rsrc(reinterpret_cast<const void*>(p - low), ((int64_t)(a.M - m0) * KB + low + 3) & ~3ll);
}

// Merge of the K groups of the few-rows kernels through LDS, and stores: element 4 q + c of a block is
// row 8 q + 4 eta + c, column lane % 32.
// mend(the wave's part): what may be put right in between.
template <int TI, int NW, int KG, typename Mend>
__device__ __forceinline__ void merge_rows(const LinArgs& a, const floatx16 (&acc)[TI], floatx4* red, int m0, int n0, int wave,
                                           int lane, Mend&& mend) {
    constexpr int CW = NW / KG;
    const int lr = lane & 31, eta = lane >> 5;
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            red[((wave * TI + i) * 4 + q) * 64 + lane] =
                floatx4{acc[i][4 * q], acc[i][4 * q + 1], acc[i][4 * q + 2], acc[i][4 * q + 3]};
    mend(red + wave * TI * 256);
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(63));
    wg_barrier();
    for (int t = wave; t < CW * TI * 4; t += NW) {
        const int q = t & 3, i = (t >> 2) % TI, c2 = (t >> 2) / TI;
        floatx4 v = floatx4{};
#pragma unroll
        for (int g = 0; g < KG; ++g) v += red[(((g * CW + c2) * TI + i) * 4 + q) * 64 + lane];
        const int m = m0 + 32 * i + 8 * q + 4 * eta, n = n0 + 32 * c2 + lr;
        if (n >= a.N) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (m + e < a.M) st_y(a, m + e, n, v[e]);
    }
}

// ---------------------------------------------------------------- few rows
// Up to some hundred rows (see kKinds).  A workgroup of NW (8 or 16)
// waves makes 32 TI rows x 32 CW columns: CW = NW / KG column waves of 32 columns, for
// each of KG groups that split the K units and merge through LDS at the end (so that a
// narrow matrix keeps enough loads in flight without partial results in memory).  A wave's
// weights and their scales go from memory straight to registers, rows of x through LDS, shared
// by the column waves of a group; both D units (256 k) deep.
// With few rows bound by the weights: 32 x 126464 x 4096 takes 56 us, 4.9 TB/s of weights, one row x 4096 x
// 4096 6.7 (latency: a launch, two units a wave, the merge).  With more, by the widening next to
// the matrix instructions: exact, 64 x 24576 x 4096 19.5 us (0.66 PFLOP/s on 192 CUs; counters: vector
// instructions issue in 63% of a SIMD's cycles, the matrix unit is busy in 44%, a wave waits in 41% of its own), 1024 x
// 3584 x 18944 131 us (1.06 PFLOP/s); to bf16 14 and 71 us.
template <int F, bool EX, int TI, int NW, int KG, int D, int OCC>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(OCC, OCC)))
void linear_mx_rows_kernel(LinArgs a, int tiles_m) {
    constexpr bool F8 = F == DARD_MX_FP8;
    constexpr int CW = NW / KG, BM = 32 * TI, RB = F8 ? 256 : 128, CPR = RB / 16, RSH = F8 ? 0 : 1;
    constexpr int XB = BM * RB, NX = XB / 1024, CX = NX >= CW ? NX / CW : 1;   // 1 KB copies per unit: all, per wave
    constexpr int LW = 5;                                                     // register loads of a wave per unit
    // scales of x: chunks of CH units per group in LDS, as aligned dwords (two a unit and one more a row)
    constexpr int CH = D == 3 ? 12 : KG * TI >= 4 ? 8 : 16, SP = 2 * CH + 1, NSC = (BM * SP + CW * 64 - 1) / (CW * 64);
    static_assert(NX % CX == 0, "whole copies per wave");
    static_assert(CH % D == 0 && CH > D, "chunks end with the unrolled loop's rounds");
    static_assert(D >= 2 && (D - 1) * (CX + LW) <= 63, "vmcnt range");
    constexpr int RING = KG * D * XB, MERGE = NW * TI * 4096, ALL = RING + KG * BM * SP * 4;
    __shared__ __attribute__((aligned(16))) char smem[ALL > MERGE ? ALL : MERGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int cw = wave % CW, kg = wave / CW, lr = lane & 31, eta = lane >> 5;
    // row tiles of the same columns next to each other on one XCD: they share the weights in its L2
    const int total = gridDim.x, xcd = blockIdx.x & 7;
    const int t0 = xcd * (total >> 3) + min(xcd, total & 7) + (int)(blockIdx.x >> 3);
    const int m0 = t0 % tiles_m * BM, n0 = t0 / tiles_m * 32 * CW;
    const int units = a.KBp / 8, KB = a.K / 32, rowb = F8 ? a.K : a.K / 2;
    const int u0 = (int)((int64_t)units * kg / KG), nu = (int)((int64_t)units * (kg + 1) / KG) - u0;
    const int most = (units + KG - 1) / KG;       // iterations of the workgroup

    const __amdgpu_buffer_rsrc_t rx = rsrc(a.xc + (size_t)m0 * rowb, (int64_t)(a.M - m0) * rowb);
    int low;
    const __amdgpu_buffer_rsrc_t rs = rsrc_xs(a, m0, KB, low);
    const size_t blk = min(n0 / 32 + cw, a.nblk - 1);
    const __amdgpu_buffer_rsrc_t rw = rsrc(a.wc + blk * a.KBp * 512, (int64_t)a.KBp * 512);
    const __amdgpu_buffer_rsrc_t rws = rsrc(a.ws + blk * units * 64, (int64_t)units * 256);
    // copy j of a wave: rows (cw CX + j) RPC + lane / CPR; slot s of row r holds chunk s ^ f(r)
    constexpr int RPC = 64 / CPR;
    int xk[CX];
#pragma unroll
    for (int j = 0; j < CX; ++j) {
        const int row = (cw * CX + j) * RPC + lane / CPR;
        xk[j] = 16 * ((lane % CPR) ^ ((row >> RSH) & (CPR - 1)));
    }
    const int xrow = (cw * CX * RPC + lane / CPR) * rowb;
    char* const ring = smem + kg * D * XB;

    uint32_t* const xsc = reinterpret_cast<uint32_t*>(smem + RING) + kg * BM * SP;
    uint32_t sreg[NSC];
    auto load_scales = [&](int i) __attribute__((always_inline)) {    // the chunk from unit i of the group on
#pragma unroll
        for (int k = 0; k < NSC; ++k) {
            const int q = (k * CW + cw) * 64 + lane, row = q / SP, d = q % SP;
            const int o = ((low + row * KB) & ~3) + 8 * (u0 + i) + 4 * d;
            sreg[k] = __builtin_amdgcn_raw_buffer_load_b32(rs, row < BM && row < a.M - m0 ? o : -16, 0, 0);
        }
    };
    auto store_scales = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < NSC; ++k) {
            const int q = (k * CW + cw) * 64 + lane;
            if (q < BM * SP) xsc[q] = sreg[k];
        }
    };

    struct Regs {
        uintx4 w[4];
        uint32_t sw;
    };
    Regs rg[D];
    auto issue = [&](int i, Regs& r, int slot) __attribute__((always_inline)) {   // unit i of the group (past the last: repeated)
        const int u = u0 + (nu > 0 ? min(i, nu - 1) : 0), kb = u * RB;
        __builtin_amdgcn_sched_barrier(0);
        if (NX == CW * CX || cw < NX / CX) {
#pragma unroll
            for (int j = 0; j < CX; ++j)
                copy_lds<16>(rx, ring + slot * XB + (cw * CX + j) * 1024,
                             kb + xk[j] < rowb ? xrow + xk[j] + (kb + j * RPC * rowb) : -16, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            r.w[q] = __builtin_bit_cast(uintx4, __builtin_amdgcn_raw_buffer_load_b128(rw, 16 * lane, u * 4096 + q * 1024, 0));
        r.sw = __builtin_amdgcn_raw_buffer_load_b32(rws, 4 * lane, u * 256, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    floatx16 acc[TI][1];
#pragma unroll
    for (int i = 0; i < TI; ++i) acc[i][0] = floatx16{};
    High<TI, 1> high;
    load_scales(0);
#pragma unroll
    for (int d = 0; d + 1 < D; ++d) issue(d, rg[d], d);
    store_scales();
    // Unit i: register slot and ring slot i % D.  Once this unit's copies have landed and every wave
    // is done with the unit before (its slot is free), unit i + D - 1 is issued into that slot.
    // Younger than this unit's copies are its own register loads and D - 2 whole units.
    auto unit = [&](int i, auto dc) __attribute__((always_inline)) {
        constexpr int d = decltype(dc)::value, prev = (d + D - 1) % D;
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(LW + (D - 2) * (CX + LW)));
        wg_barrier();
        if constexpr (d == 0) {
            if (i > 0 && i % CH == 0) {   // (every wave is done with the chunk before)
                store_scales();
                __builtin_amdgcn_s_waitcnt(waitcnt_vm(63));
                wg_barrier();
            }
            if (i % CH == CH - D) load_scales(i + D);
        }
        issue(i + D - 1, rg[prev], prev);
        if (i >= nu) return;   // (a group with one unit less)
        const int u = u0 + i;
        uint32_t sx[TI];
#pragma unroll
        for (int i2 = 0; i2 < TI; ++i2) {
            const uint32_t* p = xsc + (32 * i2 + lr) * SP + 2 * (i % CH);
            const uint32_t t[3] = {p[0], p[1], p[2]};
            sx[i2] = x_scales<2>(t, low + (32 * i2 + lr) * KB, 8 * u, KB, eta);
        }
        const uint32_t sw[1] = {rg[d].sw};
        if constexpr (EX) high.add(sx, sw);
        XFrag<F> x[4][TI];
#pragma unroll
        for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int i2 = 0; i2 < TI; ++i2) {
                const int row = 32 * i2 + lr, sz = (row >> RSH) & (CPR - 1);
#pragma unroll
                for (int p = 0; p < (F8 ? 2 : 1); ++p)
                    x[h][i2].c[p] = *reinterpret_cast<const uintx4*>(
                        ring + d * XB + row * RB + 16 * (((F8 ? 4 : 2) * h + x_chunk<F, EX>(eta, p)) ^ sz));
            }
        auto step = [&](auto jc) __attribute__((always_inline)) {
            constexpr int J = decltype(jc)::value;
            const uintx4 w[1] = {rg[d].w[J]};
            mm_step<F, EX, J, TI, 1>(x[J], w, sx, sw, acc);
        };
        step(std::integral_constant<int, 0>{});
        step(std::integral_constant<int, 1>{});
        step(std::integral_constant<int, 2>{});
        step(std::integral_constant<int, 3>{});
    };
    for (int i = 0; i < most; i += D) {   // (units past the last repeat its copies and add nothing)
        unit(i, std::integral_constant<int, 0>{});
        unit(i + 1, std::integral_constant<int, 1>{});
        if constexpr (D > 2) unit(i + 2, std::integral_constant<int, (D > 2 ? 2 : 0)>{});
        if constexpr (D > 3) unit(i + 3, std::integral_constant<int, (D > 3 ? 3 : 0)>{});
    }
    // (every loaded register is used, so that the counts above hold)
#pragma unroll
    for (int d = 0; d < D; ++d) {
#pragma unroll
        for (int q = 0; q < 4; ++q) asm volatile("" ::"v"(rg[d].w[q]));
        asm volatile("" ::"v"(rg[d].sw));
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    wg_barrier();
    floatx16 sum[TI];
#pragma unroll
    for (int i = 0; i < TI; ++i) sum[i] = acc[i][0];
    merge_rows<TI, NW, KG>(a, sum, reinterpret_cast<floatx4*>(smem), m0, n0, wave, lane, [&](floatx4* red) __attribute__((always_inline)) {
        if constexpr (EX) {
            if (!__any((high.x | high.w) != 0)) return;
#pragma unroll 1
            for (int i = 0; i < TI; ++i)
                redo_scaled<TI, 1>(a, m0 + 32 * i, n0 + 32 * cw, i, 0, u0, u0 + nu, high, [&](int v, float y) {
                    reinterpret_cast<float*>(red)[((i * 4 + v / 4) * 64 + lane) * 4 + v % 4] = y;
                });
        }
    });
}

// ---------------------------------------------------------------- tiles
// Four waves own a 256 x 256 tile, a wave 128 x 128 of it.  Both operands and their scales go
// through LDS in stages of two 64-k steps, NST deep, copied straight from memory.
//   Rows of x: swizzled in 16-byte chunks by which lane of a copy fetches which chunk. Row r
//   keeps chunk c in slot c ^ f(r), f chosen so that the 16 lanes which LDS serves at once
//   (16 rows, one chunk) hit 16 different 16-byte columns of its 256.
//   Packed weights: in operand order already (1 KB per 32 rows and step).
//   Scales: a dword per row for every 128 k (two dwords are read and shifted where rows of
//   scales are not dword-aligned), and the packed dword per lane of a unit.  (Loaded into
//   registers instead, their wait would also cover every copy issued before them: loads
//   complete in order.)
// The fragments of each step are read during the step before; the barrier of a stage
// stands before its last step, where every wave holds the rest of the stage in registers. It
// publishes the next stage and frees this one for a copy.
// 8192 x 37888 x 3584 MXFP4 786 us, 2.83 PFLOP/s; 8192 x 8192 x 8192 MXFP4 367 us, 2.99, MXFP8 to bf16 446 us,
// 2.47, exact 776 us, 1.42 (the bf16 instruction's rate on random data is 1.55).
template <int F, bool EX>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1)))
void linear_mx_tile_kernel(LinArgs a, int tiles_m, int tiles_n) {
    constexpr bool F8 = F == DARD_MX_FP8;
    constexpr int TI = 4, TJ = 4, WM = 2, KS = 2, NST = F8 ? 3 : 4;
    constexpr int WN = 4 / WM, BM = 32 * TI * WM, BN = 32 * TJ * WN;
    constexpr int RB = KS * (F8 ? 64 : 32), CPR = RB / 16;   // bytes and chunks of a row of x per stage
    constexpr int RSH = RB == 64 ? 2 : 1;                    // f(row) = (row >> RSH) % CPR
    constexpr int XB = BM * RB, WB = BN * KS * 32;
    constexpr int CX = XB / 4096, CW = WB / 4096;            // 1 KB copies of a wave per stage
    constexpr int XS = XB + WB, WS = XS + 2 * BM * 4, STAGE = WS + BN * 8;   // scales: two dwords a row of x
    constexpr int NXS = 2 * BM / 64, NWS = BN / 32, CS = (NXS + NWS + 3) / 4;   // 256-byte scale copies
    static_assert(XB % 4096 == 0 && WB % 4096 == 0, "whole copies per wave");
    static_assert(NST >= 3 && (NST - 1) * (CX + CW + CS) <= 63, "vmcnt range");
    __shared__ __attribute__((aligned(16))) char smem[NST * STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN, lr = lane & 31, eta = lane >> 5;
    // Tile order: each XCD a contiguous run of an order that walks groups of eight row tiles column
    // by column, so that the tiles in flight on an XCD share rows and weights in its L2.
    const int total = tiles_m * tiles_n;
    const int id = blockIdx.x, xcd = id & 7;
    const int t = xcd * (total >> 3) + min(xcd, total & 7) + (id >> 3);
    constexpr int GM = 8;
    const int grp = t / (GM * tiles_n), in = t - grp * GM * tiles_n, gm = min(GM, tiles_m - grp * GM);
    const int m0 = (grp * GM + in % gm) * BM, n0 = in / gm * BN;
    const int units = a.KBp / 8;
    constexpr int SPU = 4 / KS;                              // stages of a unit
    const int ns = SPU * units;
    const int KB = a.K / 32, rowb = F8 ? a.K : a.K / 2;      // scales and code bytes of a row of x

    // Copies.  Reads past a descriptor's end give zeros: rows past M, and k past K by an offset
    // outside.  Copy j of a wave fetches rows (wave CX + j) RPC + lane / CPR of x.
    constexpr int RPC = 64 / CPR;
    const __amdgpu_buffer_rsrc_t rx = rsrc(a.xc + (size_t)m0 * rowb, (int64_t)(a.M - m0) * rowb);
    int xk[CX];
#pragma unroll
    for (int j = 0; j < CX; ++j) {
        const int row = (wave * CX + j) * RPC + lane / CPR;
        xk[j] = 16 * ((lane % CPR) ^ ((row >> RSH) & (CPR - 1)));
    }
    const int xrow = (wave * CX * RPC + lane / CPR) * rowb;
    const int blk0 = n0 / 32;
    const __amdgpu_buffer_rsrc_t rw = rsrc(a.wc + (size_t)blk0 * a.KBp * 512, 0xFFFFFF00ll);
    int wo[CW];                                              // byte offset of copy j's KB in the tile's panel
#pragma unroll
    for (int j = 0; j < CW; ++j) {
        const int q = wave * CW + j;                         // block q / KS of the tile, step q % KS of the stage
        wo[j] = (min(q / KS, a.nblk - 1 - blk0) * a.KBp + 2 * (q % KS)) * 512;
    }
    int low;
    const __amdgpu_buffer_rsrc_t rs = rsrc_xs(a, m0, KB, low);
    const __amdgpu_buffer_rsrc_t rws = rsrc(a.ws + (size_t)blk0 * units * 64, 0xFFFFFF00ll);
    auto copy = [&](int st, int slot) __attribute__((always_inline)) {   // stage st (past the last: repeated)
        const int s = min(st, ns - 1), kb = s * RB;
        char* dst = smem + slot * STAGE;
#pragma unroll
        for (int j = 0; j < CS; ++j) {
            const int q = j * 4 + wave;
            if (q < NXS) {
                const int d = q / (BM / 64), row = q % (BM / 64) * 64 + lane;
                const int o = ((low + row * KB) & ~3) + 4 * s + 4 * d;
                copy_lds<4>(rs, dst + XS + q * 256, row < a.M - m0 ? o : -16, 0);
            } else if (q < NXS + NWS) {
                const int b = q - NXS;
                copy_lds<4>(rws, dst + WS + b * 256, 4 * lane, (min(b, a.nblk - 1 - blk0) * units + s / SPU) * 256);
            }
        }
#pragma unroll
        for (int j = 0; j < CX; ++j)
            copy_lds<16>(rx, dst + (wave * CX + j) * 1024, kb + xk[j] < rowb ? xrow + xk[j] + (kb + j * RPC * rowb) : -16, 0);
#pragma unroll
        for (int j = 0; j < CW; ++j) copy_lds<16>(rw, dst + XB + (wave * CW + j) * 1024, 16 * lane, wo[j] + s * (KS * 1024));
    };

    floatx16 acc[TI][TJ];
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[i][j] = floatx16{};
    struct Frag {
        XFrag<F> x[TI];
        uintx4 w[TJ];
    };
    auto read = [&](Frag& f, int slot, int h) __attribute__((always_inline)) {
        const char* st = smem + slot * STAGE;
#pragma unroll
        for (int i = 0; i < TI; ++i) {
            const int row = 32 * (wm * TI + i) + lr, sz = (row >> RSH) & (CPR - 1);
#pragma unroll
            for (int p = 0; p < (F8 ? 2 : 1); ++p)
                f.x[i].c[p] = *reinterpret_cast<const uintx4*>(
                    st + row * RB + 16 * (((F8 ? 4 : 2) * h + x_chunk<F, EX>(eta, p)) ^ sz));
        }
#pragma unroll
        for (int j = 0; j < TJ; ++j)
            f.w[j] = *reinterpret_cast<const uintx4*>(st + XB + ((wn * TJ + j) * KS + h) * 1024 + 16 * lane);
    };
    High<TI, TJ> high;
    // scales of a stage: byte h of a word is that of step h
    struct Scale {
        uint32_t x[TI], w[TJ];
    };
    auto scales = [&](Scale& sc, int st, int slot) __attribute__((always_inline)) {
        const char* base = smem + slot * STAGE;
        const int s = min(st, ns - 1);
#pragma unroll
        for (int i = 0; i < TI; ++i) {
            const int row = 32 * (wm * TI + i) + lr;
            const uint32_t* p = reinterpret_cast<const uint32_t*>(base + XS) + row;
            const uint32_t d[2] = {p[0], p[BM]};
            sc.x[i] = x_scales<1>(d, low + row * KB, 4 * s, KB, eta);
        }
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(base + WS + (wn * TJ + j) * 256 + 4 * lane);
            sc.w[j] = w >> (16 * (s & 1));
        }
        if constexpr (EX) high.add(sc.x, sc.w);
    };

#pragma unroll
    for (int p = 0; p < NST; ++p) copy(p, p);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(waitcnt_vm((NST - 1) * (CX + CW)));
    wg_barrier();
    int slot = 0;
    Frag f[2];
    Scale sc;
    read(f[0], 0, 0);
    scales(sc, 0, 0);
    for (int st = 0; st < ns; ++st) {
        const int next = slot + 1 == NST ? 0 : slot + 1;
        read(f[1], slot, 1);
        mm_step<F, EX, 0, TI, TJ>(f[0].x, f[0].w, sc.x, sc.w, acc);
        __builtin_amdgcn_sched_barrier(0);
        // stage st + 1 is there (at least (NST - 2)(CX + CW) copies came after its own); every read
        // of this one is done
        __builtin_amdgcn_s_waitcnt(waitcnt_vm((NST - 2) * (CX + CW)));
        wg_barrier();
        __builtin_amdgcn_sched_barrier(0);
        copy(st + NST, slot);
        Scale sn;
        read(f[0], next, 0);
        scales(sn, st + 1, next);
        mm_step<F, EX, 1, TI, TJ>(f[1].x, f[1].w, sc.x, sc.w, acc);
        __builtin_amdgcn_sched_barrier(0);
        sc = sn;
        slot = next;
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));   // no copy lands after this point, no wave reads a stage
    wg_barrier();

    // Stores.  Element v of a lane is row 8 (v / 4) + 4 eta + v % 4, column lane % 32 of its block: a
    // wave turns 32 rows at a time through an LDS area of its own (rows padded by 8 floats, so
    // that rows four apart use other banks) and stores 16 bytes a lane, whole runs of 32 TJ
    // columns.  (Stores straight from the accumulators, 2 or 4 bytes a lane, took 30 us for a
    // 256 x 256 tile, three times its K loop at K = 3584.)
    constexpr int PITCH = 32 * TJ + 8;
    static_assert(4 * 32 * PITCH * 4 <= NST * STAGE, "the waves' areas fit the stages");
    float* const area = reinterpret_cast<float*>(smem) + wave * 32 * PITCH;
    const int nw = n0 + 32 * wn * TJ;
#pragma unroll
    for (int i = 0; i < TI; ++i) {
#pragma unroll
        for (int j = 0; j < TJ; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) area[(8 * (v / 4) + 4 * eta + v % 4) * PITCH + 32 * j + lr] = acc[i][j][v];
        const int mi = m0 + 32 * (wm * TI + i);
        if constexpr (EX) {
            if (__any((high.x | high.w) != 0)) {
#pragma unroll 1
                for (int j = 0; j < TJ; ++j)
                    redo_scaled<TI, TJ>(a, mi, nw + 32 * j, i, j, 0, units, high, [&](int v, float y) {
                        area[(8 * (v / 4) + 4 * eta + v % 4) * PITCH + 32 * j + lr] = y;
                    });
            }
        }
        if (a.bf16_out) {
            constexpr int LPR = 4 * TJ;          // lanes of a row, 8 columns each
#pragma unroll
            for (int q = 0; q < 32 * LPR / 64; ++q) {
                const int row = (q * 64 + lane) / LPR, c = 8 * (lane % LPR), m = mi + row, n = nw + c;
                const floatx4 lo = *reinterpret_cast<const floatx4*>(area + row * PITCH + c);
                const floatx4 hi = *reinterpret_cast<const floatx4*>(area + row * PITCH + c + 4);
                st_8(reinterpret_cast<bf16_t*>(a.y) + (size_t)m * a.N + n, lo, hi, m < a.M ? a.N - n : 0);
            }
        } else {
            constexpr int LPR = 8 * TJ;          // lanes of a row, 4 columns each
#pragma unroll
            for (int q = 0; q < 32 * LPR / 64; ++q) {
                const int row = (q * 64 + lane) / LPR, c = 4 * (lane % LPR), m = mi + row, n = nw + c;
                const floatx4 v = *reinterpret_cast<const floatx4*>(area + row * PITCH + c);
                st_4(reinterpret_cast<float*>(a.y) + (size_t)m * a.N + n, v, m < a.M ? a.N - n : 0);
            }
        }
    }
}

// A kernel with its tile, and what it costs (us): a round of 256 workgroups takes fixed + unit per 256 k of
// a workgroup's K range.  Fitted to a sweep of all kernels (and four that hardly pay: 32 x 128 and 64 x 64 in
// eight waves, 32 x 192 in twelve, 64 x 256 in sixteen) over M 1 to 4096, N 3584 to 126464 and K 512 to 18944; the
// choice by cost loses 2% to the best of all twelve for each size there (smaller matrices take the same
// formula and were not swept).  Columns: exact, MXFP8, MXFP4.
struct Kind {
    int rows, cols, kg, threads;
    float fixed[3], unit[3];
};
constexpr Kind kKinds[] = {
    {32, 256, 1, 512, {3.4f, 3.9f, 2.4f}, {0.91f, 0.47f, 0.49f}},
    {32, 128, 4, 1024, {3.2f, 3.4f, 2.8f}, {1.92f, 1.14f, 1.25f}},
    {32, 64, 4, 512, {3.7f, 3.6f, 3.9f}, {1.25f, 0.77f, 0.63f}},
    {32, 32, 8, 512, {3.2f, 3.6f, 4.5f}, {1.45f, 1.15f, 0.82f}},
    {64, 256, 1, 512, {5.1f, 4.8f, 2.9f}, {1.54f, 0.75f, 0.69f}},
    {64, 128, 4, 1024, {4.1f, 4.3f, 2.9f}, {3.23f, 1.73f, 1.60f}},
    {128, 256, 1, 512, {8.7f, 8.4f, 10.3f}, {3.03f, 1.59f, 1.11f}},
    {256, 256, 0, 256, {8.8f, 7.2f, 11.1f}, {5.58f, 3.34f, 2.16f}},   // the tiled kernel
};

int column_of(int format, bool exact) { return format == DARD_MX_FP4 ? 2 : exact ? 0 : 1; }

int kind_of(int column, int M, int N, int K) {
    const double units = (K / 32 + 7) / 8;
    double best = 1e300;
    int kind = 0;
    for (int i = 0; i < (int)(sizeof kKinds / sizeof kKinds[0]); ++i) {
        const Kind& k = kKinds[i];
        const double groups = std::ceil((double)M / k.rows) * std::ceil((double)N / k.cols);
        if (groups >= 1 << 22 && k.kg) continue;                 // (a grid's threads are counted in 32 bits)
        double cost = std::ceil(groups / 256) * (k.fixed[column] + std::ceil(units / (k.kg ? k.kg : 1)) * k.unit[column]);
        const double mem = (double)N * K * (17. / 32) / 3.5e6;   // (the weights' time, us)
        if (cost < mem) cost = mem + 1e-3 * cost;                // (a tie there: the least work)
        if (cost < best) {
            best = cost;
            kind = i;
        }
    }
    return kind;
}

template <int F, bool EX> void run(const LinArgs& a, hipStream_t s) {
    const int kind = kind_of(column_of(F, EX), a.M, a.N, a.K);
    const Kind& k = kKinds[kind];
    const int tm = (a.M + k.rows - 1) / k.rows, tn = (a.N + k.cols - 1) / k.cols;
    const dim3 g((unsigned)tm * tn);
    auto few = [&](auto kernel) { launch(kernel, g, dim3(k.threads), 0, s, a, tm); };
    switch (kind) {
        case 0: few(linear_mx_rows_kernel<F, EX, 1, 8, 1, EX ? 2 : 3, 4>); break;   // (depths: what the registers hold)
        case 1: few(linear_mx_rows_kernel<F, EX, 1, 16, 4, 2, 4>); break;
        case 2: few(linear_mx_rows_kernel<F, EX, 1, 8, 4, 4, 2>); break;
        case 3: few(linear_mx_rows_kernel<F, EX, 1, 8, 8, 2, 2>); break;
        case 4: few(linear_mx_rows_kernel<F, EX, 2, 8, 1, F == DARD_MX_FP8 ? 2 : 3, 4>); break;
        case 5: few(linear_mx_rows_kernel<F, EX, 2, 16, 4, 2, 4>); break;
        case 6: few(linear_mx_rows_kernel<F, EX, 4, 8, 1, 3, 2>); break;
        default: launch(linear_mx_tile_kernel<F, EX>, g, dim3(256), 0, s, a, tm, tn);
    }
}

// fp32 outputs of MXFP8 rows take the exact products: the scaled instruction's alignment leaves
// 4.5e-6 of the result (its norm), where float32 sums leave 1e-7; a bf16 output's rounding, 2e-3,
// hides it, and of E2M1 products (8 bits wide at most) none is cut.
bool exact_of(int format, int out_dtype) { return format == DARD_MX_FP8 && out_dtype == DARD_DTYPE_F32; }

}  // namespace

void linear_mx_plan(int format, int out_dtype, int M, int N, int K, int32_t* plan) {
    const bool exact = exact_of(format, out_dtype);
    const Kind& k = kKinds[kind_of(column_of(format, exact), M, N, K)];
    plan[0] = k.rows;
    plan[1] = k.cols;
    plan[2] = k.kg;
    plan[3] = exact;
}

hipError_t launch_linear_mx(int format, const uint8_t* xc, const uint8_t* xs, int M, int K, const void* Wp, int N,
                            int out_dtype, void* y, hipStream_t s) {
    const MxPacked w = mx_packed(N, K);
    LinArgs a{};
    a.xc = xc; a.xs = xs; a.wc = (const uint8_t*)Wp; a.ws = (const uint32_t*)((const char*)Wp + w.scales);
    a.M = M; a.K = K; a.N = N; a.KBp = w.KBp; a.nblk = w.nblk;
    a.bf16_out = out_dtype == DARD_DTYPE_BF16;
    a.y = y;
    if (format == DARD_MX_FP4) run<DARD_MX_FP4, false>(a, s);
    else if (exact_of(format, out_dtype)) run<DARD_MX_FP8, true>(a, s);
    else run<DARD_MX_FP8, false>(a, s);
    return hipGetLastError();
}

}  // namespace dard
