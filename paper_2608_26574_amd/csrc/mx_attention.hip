// State-masked attention over an MXFP4 key/value cache (Sec. 3.1, Sec. 3.2;
// the block-scaled form of the prefix cache of App. C.5).
//
// One pass over the keys on v_mfma_f32_32x32x16_bf16: S^T = K Q^T and O^T += V^T P^T over
// tiles of 32 keys, with a running maximum and sum per query row.  The rows of
// all query heads of a KV head are one row space.  A wave takes 32 JT rows and
// whole key tiles on its own: codes go from memory straight to its ring in LDS, in
// operand order, and are widened to bf16 in registers by the scaled conversions
// (exact: an E2M1 value times a power of two), so the main loop has no barrier.
// The four waves of a workgroup take interleaved tiles and merge
// through LDS; long key ranges are also split over workgroups (fp32 partials,
// merged in split order by a second kernel).
//
// What bounds it: per tile and 64 rows 32 matrix instructions and about 250
// others, of which 64 widen codes, 32 pair V's keys and 32 are exp2.  Counters at 448 rows and
// 131136 keys (131 us): vector instructions issue in 75% of a SIMD's cycles, the matrix
// unit is busy in 64%; a tile takes a SIMD 0.84 us (the difference of 98368 and 131136 keys).  Two
// waves a SIMD with the queries in LDS (read anew for every tile) beat one wave with them
// in registers, 133 to 170 us at that size before the order of the waves below was set, though that
// one alternates both kinds of instruction by hand.
//
// Operand order.  Lane l is row l % 32 of an operand, eta = l / 32.
//   S^T: A row i holds key pi(i), pi swapping bits 2 and 3, and a lane's dims are
//   the half eta of the head, so its codes are one contiguous run of its key.
//   The accumulator then gives a lane, for its query row, keys 16 m + 8 eta + 0..7
//   of the tile in elements 8 m .. 8 m + 7: the P^T operand of step m as it stands.
//   O^T: A row i of block t holds dim (dh/32) i + t, and the lane needs 8
//   consecutive keys of it: the cache keeps V in groups of 8 keys whose two bytes
//   per 4 dims lie together, so a lane reads its 8 keys as 16 bytes and pairs
//   neighbouring keys after the conversion.
//
// Key tiles are aligned to 32 from key 0.  Tiles below the sequence's prefix
// length are seen by every row; later ones are tested against the row's
// visibility string (one bit per block key, x then s; zero past the block).
#include <cmath>

#include "launch.h"
#include "mx.h"

namespace dard {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFloor = -3.402823466e38f;   // start of a running maximum (log2 units): the least finite score
constexpr float kBig = 256.f;      // a lane's probability sum over a tile that moves the running max
constexpr int kTileKeys = 32;
constexpr uint32_t kFarScale = 253;   // least scale code whose values can be infinite in bf16: 4 * 2^126
constexpr int kVisWords = 2 * kMaxBlock / 32 + 2;   // 32-bit words of a row's visibility, padded

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Two floats to bf16 (the hardware's conversion: nearest even, NaN stays NaN).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{lo, hi}, bf16x2));
}

// s plus both values of a pair.
__device__ __forceinline__ float add_pair(uint32_t pair, float s) {
    const bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), one, s, false);
}

__device__ __forceinline__ bf16x8 as_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_bit_cast(bf16x8, make_uint4(a, b, c, d));
}

// Codes and scales of one key tile as a lane reads them from LDS (vector types:
// reads of the uint4 struct lose the type information without which the compiler
// makes them wait for every copy in flight).
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));
template <int DH> struct RawK {
    uintx4 c[DH / 64];    // this lane's half key
    uint32_t s;           // its scales (one byte per 32 dims)
};
struct RawV {
    uintx4 c[2];          // 8 keys of this lane's dims, steps m = 0, 1
    uintx2 s[2];          // their scales
};

// A wave's ring of key tiles in LDS.  Copies run kDepth tiles ahead straight from
// memory to LDS (no registers), so a wave keeps enough loads in flight to cover the
// memory's latency on its own; the ring is the wave's alone, so its waits are counts of its
// own copies.  A slot holds every lane's operands in lane order (reads of 16
// bytes are consecutive over the lanes): K codes [DH/64][64][16], V codes
// [DH/64][64][16], then the DH bytes of K scales and the DH of V scales.
template <int DH> struct Slot {
    static constexpr int kV = DH * 16, kKs = 2 * kV, kVs = kKs + DH, kBytes = kVs + DH;
    static constexpr int kCopies = 2 * (DH / 64) + 2;
};

__device__ __forceinline__ void copy16_lds(__amdgpu_buffer_rsrc_t r, char* dst, int voff) {
#if __HIP_DEVICE_COMPILE__   // (the host pass does not know the builtin)
    typedef __attribute__((address_space(3))) void* lds_ptr;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr)dst, 16, voff, 0, 0, 0);
#endif
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const uint8_t* p) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)p, (short)0, -1, 0x00020000);
}

// Cache of one sequence and KV head, and this lane's byte offsets in a tile.
template <int DH> struct Tiles {
    const uint8_t *kc, *ks, *vc, *vs;   // at key 0
    int ko, vo, vs16;
    bool scales;                        // lanes that copy the tile's DH scale bytes
    __device__ __forceinline__ Tiles(const MxAttnArgs& a, size_t row0, int lane) {
        kc = a.kc + row0 * (DH / 2);
        ks = a.ks + row0 * (DH / 32);
        vc = a.vc + row0 * (DH / 2);
        vs = a.vs + row0 * (DH / 32);
        const int lr = lane & 31, eta = lane >> 5;
        ko = ((lr & ~12) | ((lr & 4) << 1) | ((lr & 8) >> 1)) * (DH / 2) + eta * (DH / 4);
        vo = DH == 128 ? (eta * 32 + lr) * 16 : lane * 16;
        vs16 = lane * 16;
        scales = lane < DH / 16;
    }
    __device__ __forceinline__ void copy(int t, char* slot) const {
        const __amdgpu_buffer_rsrc_t k = rsrc(kc + (size_t)t * (16 * DH)), v = rsrc(vc + (size_t)t * (16 * DH));
        const __amdgpu_buffer_rsrc_t sk = rsrc(ks + (size_t)t * DH), sv = rsrc(vs + (size_t)t * DH);
#pragma unroll
        for (int i = 0; i < DH / 64; ++i) copy16_lds(k, slot + i * 1024, ko + 16 * i);
#pragma unroll
        for (int i = 0; i < DH / 64; ++i) copy16_lds(v, slot + Slot<DH>::kV + i * 1024, vo + 1024 * i);
        __builtin_amdgcn_sched_barrier(0);
        if (scales) {   // (nothing else in here: without a branch around them the compiler's own counts of copies hold)
            copy16_lds(sk, slot + Slot<DH>::kKs, vs16);
            copy16_lds(sv, slot + Slot<DH>::kVs, vs16);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
};

template <int DH> __device__ __forceinline__ RawK<DH> read_k(const char* slot, int lane) {
    RawK<DH> t;
    const int lr = lane & 31, eta = lane >> 5, key = (lr & ~12) | ((lr & 4) << 1) | ((lr & 8) >> 1);
#pragma unroll
    for (int i = 0; i < DH / 64; ++i) t.c[i] = *reinterpret_cast<const uintx4*>(slot + i * 1024 + lane * 16);
    if constexpr (DH == 128) t.s = *reinterpret_cast<const uint16_t*>(slot + Slot<DH>::kKs + key * 4 + 2 * eta);
    else t.s = *reinterpret_cast<const uint8_t*>(slot + Slot<DH>::kKs + key * 2 + eta);
    return t;
}
template <int DH> __device__ __forceinline__ RawV read_v(const char* slot, int lane) {
    RawV t;
    const int lr = lane & 31, eta = lane >> 5;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const int grp = 2 * m + eta, blk = DH == 128 ? lr >> 3 : lr >> 4;
        t.c[m] = *reinterpret_cast<const uintx4*>(slot + Slot<DH>::kV + (DH == 128 ? m * 1024 + lane * 16 : (grp * 16 + (lr >> 1)) * 16));
        t.s[m] = *reinterpret_cast<const uintx2*>(slot + Slot<DH>::kVs + (grp * (DH / 32) + blk) * 8);
    }
    return t;
}

// Byte i of w as the scale of a conversion.  Those read a float's exponent
// field alone (checked with every other bit set and clear), so one shift does.
template <int I> __device__ __forceinline__ float scale_at(uint32_t w) {
    return __uint_as_float(I < 3 ? w << (23 - 8 * I) : w >> 1);
}

// Bits [start, start + 64) of a bit string of kBlockWords words, zero outside.
__device__ __forceinline__ uint64_t bits_at(const uint64_t* x, int start) {
    if (start <= -64 || start >= 64 * kBlockWords) return 0ull;
    if (start < 0) return x[0] << -start;
    const int q = start >> 6, sh = start & 63;
    uint64_t v = x[q] >> sh;
    if (sh && q + 1 < kBlockWords) v |= x[q + 1] << (64 - sh);
    return v;
}

// Position of workgroup `id` of `total` when the eight XCDs, which take
// workgroups in turn, each get one contiguous run.
__device__ __forceinline__ int xcd_run(int id, int total) {
    const int x = id & 7, q = total >> 3, r = total & 7;
    return x * q + min(x, r) + (id >> 3);
}

// S^T = K Q^T of one tile; q: the query operands in LDS, [JT][DH / 16][64 lanes].
template <int DH, int JT>
__device__ __forceinline__ void scores(const RawK<DH>& k, const bf16x8* q, int lane, floatx16 (&st)[JT]) {
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) st[jt] = floatx16{};
    const float f[2] = {scale_at<0>(k.s), scale_at<1>(k.s)};
#pragma unroll
    for (int j = 0; j < DH / 16; ++j) {
        const uint32_t x = k.c[j / 4][j & 3];
        const bf16x8 kf = as_bf16x8(fp4x2_to_bf16x2<0>(x, f[j / 4]), fp4x2_to_bf16x2<1>(x, f[j / 4]),
                                    fp4x2_to_bf16x2<2>(x, f[j / 4]), fp4x2_to_bf16x2<3>(x, f[j / 4]));
#pragma unroll
        for (int jt = 0; jt < JT; ++jt) st[jt] = mfma32x32x16(kf, q[(jt * (DH / 16) + j) * 64 + lane], st[jt]);
    }
}

// Probabilities of one tile against the running maximum m (log2 units, c =
// log2 units per score), which may lag the true one: a lane whose sum of them
// exceeds kBig (always on a row's first visible tile, and whenever a score is
// more than 8 above m) has the tile's maximum taken, the accumulators rescaled
// and the probabilities formed again, so other tiles need no maximum.
// They are rounded to bf16, the type in which the matrix instruction takes
// them (as in the framework's bf16 attention), and the row sum, in float32, is that of the rounded ones, so that the
// weights add up to 1.  On ordinary data the result is then off by 0.0021 to 0.0023 of its norm, where the
// bf16 output alone leaves 0.0017.
template <int JT, int NT>
__device__ __forceinline__ void probabilities(const floatx16 (&st)[JT], float c, float (&m)[JT], float (&l)[JT],
                                              floatx16 (&o)[JT][NT], uint32_t (&p)[JT][8]) {
    float sum[JT];
    auto form = [&](int jt) __attribute__((always_inline)) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float p0 = exp2_fast(fmaf(st[jt][2 * e], c, -m[jt])), p1 = exp2_fast(fmaf(st[jt][2 * e + 1], c, -m[jt]));
            p[jt][e] = pack_bf16(p0, p1);
            if (e & 1) b = add_pair(p[jt][e], b);
            else a = add_pair(p[jt][e], a);
        }
        sum[jt] = a + b;
    };
    bool big = false;
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) {
        form(jt);
        big |= sum[jt] > kBig;
    }
    if (__builtin_expect(__any(big), 0)) {
#pragma unroll
        for (int jt = 0; jt < JT; ++jt) {
            float top = st[jt][0];
#pragma unroll
            for (int e = 1; e < 16; ++e) top = fmaxf(top, st[jt][e]);
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float mn = fmaxf(m[jt], top * c);
            const float al = exp2_fast(m[jt] - mn);
            m[jt] = mn;
            l[jt] *= al;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[jt][t][e] *= al;
            form(jt);
        }
    }
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) l[jt] += sum[jt];
}

// O^T += V^T P^T of one tile.
template <int DH, int JT>
__device__ __forceinline__ void add_values(const RawV& v, const uint32_t (&p)[JT][8], int lr, floatx16 (&o)[JT][DH / 32]) {
    constexpr int NT = DH / 32;
#pragma unroll
    for (int mm = 0; mm < 2; ++mm) {
        uint32_t vf[NT][4];
        const float f[8] = {scale_at<0>(v.s[mm].x), scale_at<1>(v.s[mm].x), scale_at<2>(v.s[mm].x), scale_at<3>(v.s[mm].x),
                            scale_at<0>(v.s[mm].y), scale_at<1>(v.s[mm].y), scale_at<2>(v.s[mm].y), scale_at<3>(v.s[mm].y)};
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // keys 2 i, 2 i + 1
            if constexpr (DH == 128) {
                const uint32_t a0 = fp4x2_to_bf16x2<0>(v.c[mm][i], f[2 * i]), a1 = fp4x2_to_bf16x2<1>(v.c[mm][i], f[2 * i]);
                const uint32_t b0 = fp4x2_to_bf16x2<2>(v.c[mm][i], f[2 * i + 1]), b1 = fp4x2_to_bf16x2<3>(v.c[mm][i], f[2 * i + 1]);
                vf[0][i] = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
                vf[1][i] = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
                vf[2][i] = __builtin_amdgcn_perm(b1, a1, 0x05040100u);
                vf[3][i] = __builtin_amdgcn_perm(b1, a1, 0x07060302u);
            } else {
                const uint32_t x = v.c[mm][i] >> (8 * (lr & 1));   // this lane's two dims of the four
                const uint32_t a0 = fp4x2_to_bf16x2<0>(x, f[2 * i]), b0 = fp4x2_to_bf16x2<2>(x, f[2 * i + 1]);
                vf[0][i] = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
                vf[1][i] = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int jt = 0; jt < JT; ++jt)
                o[jt][t] = mfma32x32x16(as_bf16x8(vf[t][0], vf[t][1], vf[t][2], vf[t][3]),
                                        as_bf16x8(p[jt][4 * mm], p[jt][4 * mm + 1], p[jt][4 * mm + 2], p[jt][4 * mm + 3]),
                                        o[jt][t]);
    }
}

// O^T += what key j of a tile adds through its V blocks of large scales (bit j of far[b], b the block of 32 dims), in the rows
// that see it (bit j of seen).
template <int DH, int JT>
__device__ __forceinline__ void add_far(const char* slot, int j, const uint32_t (&far)[DH / 32], const uint32_t (&seen)[JT],
                                        const uint32_t (&p)[JT][8], int lr, int eta, floatx16 (&o)[JT][DH / 32]) {
    constexpr int NT = DH / 32;
    const uint8_t* const vc = reinterpret_cast<const uint8_t*>(slot) + Slot<DH>::kV + (j >> 3) * (4 * DH) + 2 * (j & 7);
    const uint8_t* const vs = reinterpret_cast<const uint8_t*>(slot) + Slot<DH>::kVs + (j >> 3) * (DH / 4) + (j & 7);
    float w[JT];   // key j's probability: element 8 (j / 16) + j % 8 of the lanes of half j / 8 % 2
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) {
        uint32_t pair = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) pair = e == 4 * (j >> 4) + (j & 7) / 2 ? p[jt][e] : pair;
        pair = (uint32_t)__shfl((int)pair, lr + 32 * ((j >> 3) & 1), 64);
        w[jt] = __uint_as_float(j & 1 ? pair & 0xFFFF0000u : pair << 16);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int b = (e / 4) * NT / 4, row = 8 * (e / 4) + 4 * eta + e % 4;   // A row: dims NT row .. NT row + NT - 1
        if (((far[b] >> j) & 1u) == 0) continue;
        const float f = mx_scale_f(vs[8 * b]);
        const uint32_t x = NT == 4 ? (uint32_t)*reinterpret_cast<const uint16_t*>(vc + 16 * row) : (uint32_t)vc[16 * (row / 2) + row % 2];
#pragma unroll
        for (int t = 0; t < NT; t += 2) {
            const uint32_t v = t ? fp4x2_to_bf16x2<1>(x, f) : fp4x2_to_bf16x2<0>(x, f);
#pragma unroll
            for (int jt = 0; jt < JT; ++jt) {
                if (((seen[jt] >> j) & 1u) == 0) continue;
                o[jt][t][e] = fmaf(w[jt], __uint_as_float(v << 16), o[jt][t][e]);
                o[jt][t + 1][e] = fmaf(w[jt], __uint_as_float(v & 0xFFFF0000u), o[jt][t + 1][e]);
            }
        }
    }
}

template <int DH, int JT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attn_mx_kernel(MxAttnArgs a, int rowtiles, int tps) {
    constexpr int NJ = DH / 16, NT = DH / 32;
    constexpr int kDepth = DH == 128 ? 3 : 5;          // tiles in flight per wave (two workgroups share a CU)
    constexpr int kRing = kDepth * Slot<DH>::kBytes;
    static_assert(kDepth * Slot<DH>::kCopies <= 63, "vmcnt range");
    constexpr int kMerge = NT * 4 * 64 * 16;           // O of one row tile of a wave
    // One array (several would carry alias information by which the compiler makes every LDS read
    // wait for every copy in flight): the rings and the query operands, in whose place O of one row
    // tile of the four waves lies at the end; the waves' maxima and sums; the rows' take-x words and their
    // complements; the rows' visibility strings.
    constexpr int kQ = 4 * kRing, kMl = kQ + JT * NJ * 1024 > 4 * kMerge ? kQ + JT * NJ * 1024 : 4 * kMerge;
    constexpr int kXs = kMl + 4 * JT * 64 * 4, kVis = kXs + 32 * JT * 2 * kBlockWords * 8;
    __shared__ __attribute__((aligned(16))) char smem[kVis + 32 * JT * kVisWords * 4];
    float* const ml = reinterpret_cast<float*>(smem + kMl);
    uint64_t* const xs = reinterpret_cast<uint64_t*>(smem + kXs);
    uint64_t* const vis = reinterpret_cast<uint64_t*>(smem + kVis);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane & 31, eta = lane >> 5;
    const int nsplit = gridDim.y;
    int id = xcd_run(blockIdx.y * gridDim.x + blockIdx.x, gridDim.x * nsplit);
    const int rt = id % rowtiles;
    id /= rowtiles;
    const int split = id % nsplit;
    id /= nsplit;
    const int kvh = id % a.Hkv, s = id / a.Hkv;
    const int R = 2 * a.B, GQ = a.Hq / a.Hkv, nrows = GQ * R;
    int P = a.P;
    if (a.prefix) P = min(max(__builtin_amdgcn_readfirstlane(a.prefix[s]), 0), a.P);
    const int nkeys = P + R, ntiles = (nkeys + kTileKeys - 1) / kTileKeys;
    const int t0 = split * tps, t1 = min(ntiles, t0 + tps);

    // query operands of the row tile, which the waves share: operand (jt, j), for lane l, holds row
    // 32 jt + l % 32, the 8 dims from 8 j on of the half l / 32
    bf16x8* const q = reinterpret_cast<bf16x8*>(smem + kQ);
    bf16x8 qv[JT * NJ / 4];
#pragma unroll
    for (int i = 0; i < JT * NJ / 4; ++i) {
        const int jt = (4 * i + wave) / NJ, j = (4 * i + wave) % NJ;
        const int rho = min(rt * 32 * JT + 32 * jt + lr, nrows - 1);
        qv[i] = ld_bf16x8(a.q + (((size_t)s * R + rho % R) * a.Hq + kvh * GQ + rho / R) * DH + eta * (DH / 2) + 8 * j);
    }
    // states and confidences: of a row of the tile, and of a block position of word `wave`
    const bool block = t1 * kTileKeys > P && t0 < t1;   // (the same for the workgroup)
    const int row = rt * 32 * JT + (JT == 2 ? lane : lr), r = min(row, nrows - 1) % R;
    const bool shadow = r >= a.B;
    const int pos = shadow ? r - a.B : r, wpos = 64 * wave + lane;
    int si = 0, sj = -1;
    float ci = 0.f, cj = 0.f;
    if (block) {
        const uint8_t* state = a.state + (size_t)s * a.B;
        const float* conf = a.conf + (size_t)s * a.B;
        si = state[pos];
        ci = conf[pos];
        if (wpos < a.B) {
            sj = state[wpos];
            cj = conf[wpos];
        }
    }
    __builtin_amdgcn_sched_barrier(0);   // (these loads before the rings' copies: waits are in order)
    const size_t row0 = ((size_t)s * a.Hkv + kvh) * a.cap;
    // this wave's tiles: t0 + wave + 4 i for i < n, the first `full` of them seen whole by
    // every row.  Tile i sits in ring slot i % kDepth; copies past the last repeat it, so that the
    // number in flight is always the same.
    const Tiles<DH> tiles(a, row0, lane);
    char* ring = smem + wave * kRing;
    const int first = t0 + wave, n = max(0, (t1 - first + 3) >> 2);
    const int full = max(0, (min(t1, P / kTileKeys) - first + 3) >> 2);
    int at = 0;            // ring slot of tile i
    auto next_slot = [&](int x) { return x + 1 == kDepth ? 0 : x + 1; };
#pragma unroll
    for (int i = 0; i < kDepth; ++i)
        tiles.copy(min(first + 4 * min(i, max(n - 1, 0)), ntiles - 1), ring + i * Slot<DH>::kBytes);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < JT * NJ / 4; ++i) q[(4 * i + wave) * 64 + lane] = qv[i];
    // Visibility strings of the workgroup's rows, where its keys reach the block: wave w forms the
    // 64 positions from 64 w on of every row (a lane per row).  The rules are those of take_x:
    // ballots give the U and C sets, a candidate row compares its confidence with every candidate's.
    if (block) {
        const uint64_t U = __ballot(sj == DARD_STATE_U), C = __ballot(sj == DARD_STATE_C);
        const uint64_t in = block_word_mask(a.B, wave), self = (pos >> 6) == wave ? 1ull << (pos & 63) : 0ull;
        uint64_t better = C;
        if (a.flags & DARD_F_ORDER_L2R) {
            const int upto = pos - 64 * wave + 1;   // positions of this word that are <= pos
            better &= upto >= 64 ? ~0ull : (upto <= 0 ? 0ull : (1ull << upto) - 1);
        } else if (!(a.flags & DARD_F_C_BIDIR)) {
            better = 0ull;
            for (uint64_t left = C; left; left &= left - 1) {
                const int j = __builtin_ctzll(left);
                const float x = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(cj), j));
                better |= ci <= x ? 1ull << j : 0ull;
            }
        }
        uint64_t x;
        if (si == DARD_STATE_U) x = (shadow || (a.flags & DARD_F_XSELF_SHADOW)) ? U & ~self : U;
        else if (si == DARD_STATE_C) x = shadow ? (U | better) & ~self : U | better;
        else if (shadow) x = U;
        else x = (a.flags & DARD_F_MKEYS_SHADOW) ? U | C | self : in;
        if (JT == 2 || eta == 0) {
            xs[(JT == 2 ? lane : lr) * 2 * kBlockWords + wave] = x;
            xs[(JT == 2 ? lane : lr) * 2 * kBlockWords + kBlockWords + wave] = ~x & in;
        }
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(63));
        wg_barrier();
        // bit j of a row's string: key j of the block, x keys (bits of x), then s keys (the others).  The
        // words that tiles up to the block's end read: the last one from bit 2 B - 1 at most.
        for (int i = threadIdx.x; i < 32 * JT * ((2 * a.B + 31) / 64 + 1); i += 256) {
            const int at = i % (32 * JT), word = i / (32 * JT), start = 64 * word;
            const uint64_t* w = xs + at * 2 * kBlockWords;
            vis[at * (kVisWords / 2) + word] = bits_at(w, start) | bits_at(w + kBlockWords, start - a.B);
        }
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(63));
    wg_barrier();

    const float c = a.scale * kLog2e;
    floatx16 o[JT][NT];
    float m[JT], l[JT];
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) {
        m[jt] = kFloor;
        l[jt] = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) o[jt][t] = floatx16{};
    }

    auto refill = [&](int i) __attribute__((always_inline)) {   // tile i's slot, once its values are in registers
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(63));
        tiles.copy(first + 4 * min(i + kDepth, n - 1), ring + at * Slot<DH>::kBytes);
        at = next_slot(at);
    };
    int i = 0;
    for (; i < full; ++i) {
        __builtin_amdgcn_s_waitcnt(waitcnt_vm((kDepth - 1) * Slot<DH>::kCopies));   // tile i is there
        __builtin_amdgcn_sched_barrier(0);
        const RawK<DH> k = read_k<DH>(ring + at * Slot<DH>::kBytes, lane);
        const RawV v = read_v<DH>(ring + at * Slot<DH>::kBytes, lane);
        floatx16 st[JT];
        uint32_t p[JT][8];
        scores<DH, JT>(k, q, lane, st);
        probabilities<JT, NT>(st, c, m, l, o, p);
        // the wave that has its probabilities goes first: its matrix instructions run under the other
        // wave's vector ones (448 rows, 131136 keys: 135 -> 130 us; first with the scores too 133, with the
        // probabilities 136)
        __builtin_amdgcn_s_setprio(1);
        add_values<DH, JT>(v, p, lr, o);
        __builtin_amdgcn_s_setprio(0);
        refill(i);
    }
    // tiles at the prefix's end and in the block
    for (; i < n; ++i) {
        const int k0 = (first + 4 * i) * kTileKeys;
        __builtin_amdgcn_s_waitcnt(waitcnt_vm((kDepth - 1) * Slot<DH>::kCopies));
        __builtin_amdgcn_sched_barrier(0);
        const RawK<DH> k = read_k<DH>(ring + at * Slot<DH>::kBytes, lane);
        RawV v = read_v<DH>(ring + at * Slot<DH>::kBytes, lane);
        floatx16 st[JT];
        uint32_t p[JT][8], seen[JT];
        scores<DH, JT>(k, q, lane, st);
        // element 8 m + e of a lane is key k0 + 16 m + 8 eta + e
        const int j0 = k0 - P;
#pragma unroll
        for (int jt = 0; jt < JT; ++jt) {
            const uint32_t* vw = reinterpret_cast<const uint32_t*>(vis) + (32 * jt + lr) * kVisWords;
            uint32_t bits;
            if (j0 < 0) {
                bits = (vw[0] << -j0) | ((1u << -j0) - 1u);   // (-j0 < 32)
            } else {
                const int w = j0 >> 5, sh = j0 & 31;
                bits = sh ? (vw[w] >> sh) | (vw[w + 1] << (32 - sh)) : vw[w];
            }
            seen[jt] = bits;
#pragma unroll
            for (int e = 0; e < 16; ++e)
                st[jt][e] = (bits >> (16 * (e / 8) + 8 * eta + e % 8)) & 1u ? st[jt][e] : -INFINITY;
        }
        // A V block whose values may be infinite in bf16 (scale codes from kFarScale on) or are NaN would reach rows
        // that do not see its key: 0 * infinity is NaN.  The matrix instructions read it with the least scale, and
        // what it adds follows apart, row by row, for the keys of the sequence (bytes past them may be anything).
        uint32_t far[NT], mine = 0;
#pragma unroll
        for (int mm = 0; mm < 2; ++mm) {
            uint32_t sc[2] = {v.s[mm].x, v.s[mm].y};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (((sc[e / 4] >> (8 * (e & 3))) & 255u) >= kFarScale) {
                    mine |= 1u << (16 * mm + 8 * eta + e);
                    sc[e / 4] &= ~(255u << (8 * (e & 3)));
                }
            }
            v.s[mm] = uintx2{sc[0], sc[1]};
        }
        uint32_t keys = 0;   // those with such a block
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            const int src = b * (32 / NT);
            far[b] = (uint32_t)__shfl((int)mine, src, 64) | (uint32_t)__shfl((int)mine, src + 32, 64);
            keys |= far[b];
        }
        probabilities<JT, NT>(st, c, m, l, o, p);
        add_values<DH, JT>(v, p, lr, o);
        keys = (uint32_t)__builtin_amdgcn_readfirstlane((int)keys) & (nkeys - k0 >= 32 ? ~0u : (1u << (nkeys - k0)) - 1u);
#pragma unroll 1
        for (; keys; keys &= keys - 1) add_far<DH, JT>(ring + at * Slot<DH>::kBytes, __builtin_ctz(keys), far, seen, p, lr, eta, o);
        refill(i);
    }
    __builtin_amdgcn_s_waitcnt(0);   // no copy lands after this point

    // merge of the four waves
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) {
        l[jt] += __shfl_xor(l[jt], 32, 64);
        if (eta == 0) {
            ml[(wave * JT + jt) * 64 + lr] = m[jt];
            ml[(wave * JT + jt) * 64 + 32 + lr] = l[jt];
        }
    }
    floatx4* buf = reinterpret_cast<floatx4*>(smem);
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) {
        __syncthreads();
#pragma unroll
        for (int t2 = 0; t2 < NT; ++t2)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                buf[((wave * NT + t2) * 4 + v) * 64 + lane] =
                    floatx4{o[jt][t2][4 * v], o[jt][t2][4 * v + 1], o[jt][t2][4 * v + 2], o[jt][t2][4 * v + 3]};
        __syncthreads();
        float mm = kFloor, f[4], ll = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) mm = fmaxf(mm, ml[(w * JT + jt) * 64 + lr]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            f[w] = exp2_fast(ml[(w * JT + jt) * 64 + lr] - mm);
            ll += ml[(w * JT + jt) * 64 + 32 + lr] * f[w];
        }
        // this wave: rows i = 8 wave + 4 eta + 0..3 of every block: dims NT (8 wave + 4 eta) + 0 .. 4 NT - 1
        float r[4][NT];
#pragma unroll
        for (int t2 = 0; t2 < NT; ++t2) {
            floatx4 x = floatx4{};
#pragma unroll
            for (int w = 0; w < 4; ++w) x += buf[((w * NT + t2) * 4 + wave) * 64 + lane] * f[w];
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e][t2] = x[e];
        }
        const int rho = rt * 32 * JT + 32 * jt + lr;
        if (rho >= nrows) continue;
        const size_t row = ((size_t)s * R + rho % R) * a.Hq + kvh * GQ + rho / R;
        const int d0 = NT * (8 * wave + 4 * eta);
        if (nsplit == 1) {
            const float inv = 1.f / ll;
            uint32_t w[2 * NT];
#pragma unroll
            for (int i = 0; i < 2 * NT; ++i)
                w[i] = pack_bf16(r[2 * i / NT][2 * i % NT] * inv, r[(2 * i + 1) / NT][(2 * i + 1) % NT] * inv);
            uint4* dst = reinterpret_cast<uint4*>(a.out + row * DH + d0);
#pragma unroll
            for (int i = 0; i < NT / 2; ++i) dst[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        } else {
            const size_t total = (size_t)a.b * R * a.Hq, at = (size_t)split * total + row;
            float* dst = a.part + at * DH + d0;
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                floatx4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = r[(4 * i + e) / NT][(4 * i + e) % NT];
                *reinterpret_cast<floatx4*>(dst + 4 * i) = x;
            }
            if (wave == 0 && eta == 0) {
                float* pm = a.part + (size_t)nsplit * total * DH + at * 2;
                pm[0] = mm;
                pm[1] = ll;
            }
        }
    }
}

// Merge of the key splits.  DH / 4 lanes take a row, 4 dims each; lane g also fetches the maximum and sum of
// split g (g + DH / 4, ...) for all of them, so that a row costs two dependent reads
// and not two per split: the reads of a row's partial results go out eight at a time.
template <int DH>
__global__ __launch_bounds__(256) void attn_mx_combine_kernel(const float* __restrict__ part, int nsplit, int64_t rows,
                                                              bf16_t* __restrict__ out) {
    constexpr int G = DH / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int g = threadIdx.x % G;
    const int64_t row = i / G < rows ? i / G : rows - 1;   // (every lane takes part in the exchanges)
    const float* ml = part + nsplit * rows * DH + 2 * row;
    const floatx4* px = reinterpret_cast<const floatx4*>(part + row * DH) + g;
    float mm = kFloor;
    for (int s = g; s < nsplit; s += G) mm = fmaxf(mm, ml[2 * s * rows]);
#pragma unroll
    for (int d = G / 2; d > 0; d /= 2) mm = fmaxf(mm, __shfl_xor(mm, d, 64));
    floatx4 x = floatx4{};
    float l = 0.f;
    for (int s0 = 0; s0 < nsplit; s0 += G) {
        const int s = s0 + g;
        float f = 0.f;
        if (s < nsplit) {
            f = exp2_fast(ml[2 * s * rows] - mm);
            l += ml[2 * s * rows + 1] * f;
        }
        const int n = min(G, nsplit - s0);
        for (int k = 0; k < n; k += 8) {
            floatx4 t[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) t[e] = px[min(s0 + k + e, nsplit - 1) * rows * G];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float w = __shfl(f, (k + e) % G, G);   // (0 past the last split)
                if (k + e < n) x += t[e] * w;
            }
        }
    }
#pragma unroll
    for (int d = G / 2; d > 0; d /= 2) l += __shfl_xor(l, d, 64);
    const float inv = 1.f / l;
    if (i / G < rows)
        reinterpret_cast<uint2*>(out)[i] = make_uint2(pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv));
}

constexpr int kSlots = 512;   // workgroups at once: two on each of 256 CUs

struct Plan {
    int jt, rowtiles, split, tps;
};

// Keys are split over the workgroups when that is cheaper than the merge.  Costs in us, fitted to a sweep of splits
// 1 to 32 over 3 head layouts, 1 to 8 sequences, blocks of 1 to 64 and prefixes of 60 to 40000 (the
// split of least cost loses 0.4% to the best): a tile of a wave costs `alone` when its workgroup has a CU to
// itself and `shared` when two share one; a full chip starts 2.6 later than an empty one, a further
// round of workgroups 2.7; the merge takes 2.5, 0.05 a split and 0.2 a megabyte of partial results.
Plan plan_of(int b, int B, int Hq, int Hkv, int dh, int P) {
    Plan p;
    const int nrows = Hq / Hkv * 2 * B;
    p.jt = nrows > 32 ? 2 : 1;
    p.rowtiles = (nrows + 32 * p.jt - 1) / (32 * p.jt);
    const int ntiles = (P + 2 * B + kTileKeys - 1) / kTileKeys;
    const double wgs = (double)p.rowtiles * Hkv * b, mb = 8e-6 * b * 2 * B * Hq * dh;
    const double alone = p.jt == 2 ? (dh == 128 ? 1.0 : 0.78) : dh == 128 ? 0.65 : 0.51;
    const double shared = p.jt == 2 ? (dh == 128 ? 1.77 : 1.44) : dh == 128 ? 1.18 : 0.96;
    static const int kSplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128};
    double best = 1e300;
    for (int split : kSplits) {
        const int tps = (ntiles + split - 1) / split, n = (ntiles + tps - 1) / tps;
        const double all = wgs * n, rounds = std::ceil(all / kSlots);
        double cost = (tps + 3) / 4 * rounds * (all <= kSlots / 2 ? alone : shared) + 2.7 * (rounds - 1) +
                      2.6 * (all < kSlots ? all / kSlots : 1.0);
        if (n > 1) cost += 2.5 + 0.05 * n + mb * n * 0.2;
        if (cost < best) {
            best = cost;
            p.split = n;
            p.tps = tps;
        }
    }
    return p;
}

template <int DH, int JT> void run(const MxAttnArgs& a, const Plan& p, hipStream_t s) {
    launch(attn_mx_kernel<DH, JT>, dim3((unsigned)(p.rowtiles * a.Hkv * a.b), p.split), dim3(256), 0, s, a, p.rowtiles, p.tps);
}

}  // namespace

size_t attention_mx_partial_bytes(int b, int B, int Hq, int Hkv, int dh, int P) {
    const Plan p = plan_of(b, B, Hq, Hkv, dh, P);
    return p.split > 1 ? (size_t)p.split * b * 2 * B * Hq * (dh + 2) * 4 : 0;
}

hipError_t launch_attention_mx(const MxAttnArgs& a, hipStream_t s) {
    const Plan p = plan_of(a.b, a.B, a.Hq, a.Hkv, a.dh, a.P);
    if (a.dh == 128) {
        if (p.jt == 2) run<128, 2>(a, p, s);
        else run<128, 1>(a, p, s);
    } else {
        if (p.jt == 2) run<64, 2>(a, p, s);
        else run<64, 1>(a, p, s);
    }
    if (p.split > 1) {
        const int64_t rows = (int64_t)a.b * 2 * a.B * a.Hq;
        const dim3 gc((unsigned)((rows * (a.dh / 4) + 255) / 256));
        if (a.dh == 128) launch(attn_mx_combine_kernel<128>, gc, dim3(256), 0, s, a.part, p.split, rows, a.out);
        else launch(attn_mx_combine_kernel<64>, gc, dim3(256), 0, s, a.part, p.split, rows, a.out);
    }
    return hipGetLastError();
}

}  // namespace dard
