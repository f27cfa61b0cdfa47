// Which keys of a cache get attention, and the cache cut to those that do:
// the softmax weight of every key summed over the rows that read it
// (dard_key_weights), the keys with the largest sums (dard_kv_select) and the
// compaction of K, V and the sums to them (dard_kv_compact).  The prefix cache is
// that of App. C.5.
#include <algorithm>
#include <type_traits>

#include "attention_tiles.h"
#include "common.h"
#include "launch.h"

namespace dard {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4e __attribute__((aligned(4)));            // at an fp32 element's alignment

__device__ __forceinline__ int prefix_len(const int32_t* prefix, int s, int P) {
    return prefix ? min(max(prefix[s], 0), P) : P;
}

// ---------------------------------------------------------------- key weights
// W_j = decay W_j + sum_r e^(scale q_r . k_j - L_r) over the rows r of all query
// heads of the KV head, L_r the row's log softmax sum.
//
// S^T = K Q^T on v_mfma_f32_32x32x16_bf16 with the keys in registers (one or two
// blocks of 32 a wave, KB) and the rows streamed through LDS, 64 at a time, so a lane
// holds one row and 16 keys of each block: L_r is one register, a score costs a
// multiply-add, an exp2 and an addition, and lanes are summed once, at the end.  Rows are
// split over workgroups where keys alone are too few (partial sums in memory, added in
// order).  Bound by those three instructions: 7168 rows x 4 heads of 128, 16384 keys 135
// us, vector instructions issue in 66 % of a SIMD's cycles (the exponential takes four
// times a multiply-add), the matrix unit is busy in 41 %.  64 rows of 16 x 32 heads, FP8,
// up to 1664 keys (rows in registers, below) 23 us, 2.8 TB/s; 64 rows x 32 heads, 609 keys
// 6.6 us.
constexpr int kWRows = 64;       // rows of a stage

// A workgroup's (sequence, KV head), key tile and row split: splits fastest, then
// key tiles, dealt to the XCDs in contiguous runs, so those that read the same rows
// share an L2; heads go to the runs in turn where they divide by 8, so that every
// XCD has heads of every sequence, however their lengths differ.
struct WeightUnit {
    int head, kt, split;
};
__device__ __forceinline__ WeightUnit weight_unit(const KeyWeightArgs& a, int nsplit, int tile) {
    const int total = gridDim.x, x = blockIdx.x & 7, ktiles = (a.P + tile - 1) / tile, heads = a.b * a.Hkv;
    const int bid = x * (total >> 3) + min(x, total & 7) + (blockIdx.x >> 3);
    const int slot = bid / nsplit / ktiles, per = heads >> 3;
    return {heads & 7 ? slot : slot % per * 8 + slot / per, bid / nsplit % ktiles, bid % nsplit};
}

// decay = 0 does not read the old sum (it may hold anything).
__device__ __forceinline__ void add_weight(const KeyWeightArgs& a, int head, int key, float x) {
    float* w = a.weights + (size_t)head * a.ldw + key;
    *w = a.decay == 0.f ? x : fmaf(a.decay, *w, x);
}

// Sums of 16 values over the 32 lanes of a half wave: each exchange halves the
// values that a lane carries, so 16 shuffles do what 80 would.  Lanes 2v and 2v + 1
// return value v.
__device__ __forceinline__ float half_sums(const float (&x)[16], int lr) {
    float y[8];
#pragma unroll
    for (int v = 0; v < 8; ++v) {
        const bool up = lr & 16;
        y[v] = (up ? x[v + 8] : x[v]) + __shfl_xor(up ? x[v] : x[v + 8], 16, 64);
    }
#pragma unroll
    for (int o = 8, n = 4; n >= 1; o >>= 1, n >>= 1) {
        const bool up = lr & o;
#pragma unroll
        for (int v = 0; v < n; ++v) {
            const float give = up ? y[v] : y[v + n], have = up ? y[v + n] : y[v];
            y[v] = have + __shfl_xor(give, o, 64);
        }
    }
    return y[0] + __shfl_xor(y[0], 1, 64);
}

template <int DH, int KB, bool KV8>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(KB == 1 ? 4 : 2)))
void key_weights_kernel(KeyWeightArgs a, int nsplit) {
    constexpr int NC = DH / 16, CH = DH / 8;                 // MFMA steps; 16-byte chunks of a row
    constexpr int STAGE = kWRows * DH * 2, NI = kWRows * CH / 256, HALVES = kWRows / 32;
    __shared__ __attribute__((aligned(16))) char smem[2 * STAGE];
    typedef __attribute__((address_space(3))) void* lds_ptr;
    typedef __attribute__((address_space(1))) void* glb_ptr;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lr = lane & 31, eta = lane >> 5;
    const WeightUnit un = weight_unit(a, nsplit, 128 * KB);
    const int g = un.head % a.Hkv, s = un.head / a.Hkv, kt = un.kt, split = un.split;
    const int p = prefix_len(a.prefix, s, a.P), k0 = (kt * 4 + wave) * 32 * KB;
    if (kt * 128 * KB >= p) return;
    const int GQ = a.Hq / a.Hkv, rows = GQ * a.R;
    const int ntile = (rows + kWRows - 1) / kWRows;
    const int t0 = (int)((long long)ntile * split / nsplit), t1 = (int)((long long)ntile * (split + 1) / nsplit);

    // this wave's keys: A operand row lr of block kb; a key past the last one repeats it.
    // Step c of an operand takes chunk ch(c, eta) of its row (any order will do that K and
    // Q share; this one makes a lane's FP8 codes of two steps 16 neighbouring bytes)
    auto ch = [&](int c) __attribute__((always_inline)) { return 4 * (c >> 1) + 2 * eta + (c & 1); };
    bf16x8 kf[KB][NC];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
        const size_t key = min(k0 + 32 * kb + lr, p - 1);
        const size_t row = (((size_t)s * a.Hkv + g) * a.cap + key) * DH;
        if constexpr (KV8) {
#pragma unroll
            for (int c = 0; c < NC; c += 2) {
                const uint4 w = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(a.k) + row + 8 * ch(c));
                kf[kb][c] = __builtin_bit_cast(bf16x8, e4m3x8_to_bf16x8_scaled(w.x, w.y));
                kf[kb][c + 1] = __builtin_bit_cast(bf16x8, e4m3x8_to_bf16x8_scaled(w.z, w.w));
            }
        } else {
#pragma unroll
            for (int c = 0; c < NC; ++c) kf[kb][c] = ld_bf16x8(reinterpret_cast<const bf16_t*>(a.k) + row + 8 * ch(c));
        }
    }

    // rows in the order (position row, head): GQ neighbours in memory.  A stage's first
    // row is divided once, a row of it by multiplication (rem + i < GQ + 64, GQ <= 32768)
    const bf16_t* qb = reinterpret_cast<const bf16_t*>(a.q) + ((size_t)s * a.R * a.Hq + (size_t)g * GQ) * DH;
    const float* lb = a.lse + (size_t)s * a.R * a.Hq + (size_t)g * GQ;
    const uint32_t magic = GQ > 1 ? 0xFFFFFFFFu / (uint32_t)GQ + 1u : 0u;
    auto row_at = [&](int pos, int rem, int i) __attribute__((always_inline)) {
        const uint32_t x = rem + i, d = GQ > 1 ? __umulhi(x, magic) : x;
        return (size_t)(pos + (int)d) * a.Hq + (x - d * GQ);
    };
    // chunk c of row r sits in slot c ^ swizzle(r): the operand reads of 16 lanes hit different banks
    auto swz = [&](int r) __attribute__((always_inline)) { return CH == 16 ? r & 15 : (r ^ (r >> 3)) & 7; };
    float L[HALVES];
    auto issue = [&](int t, char* dst) __attribute__((always_inline)) {
        const int pos = t * kWRows / GQ, rem = t * kWRows % GQ, most = rows - 1 - t * kWRows;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int q = (wave * NI + j) * 64 + lane, r = q / CH, c = (q % CH) ^ swz(r);
            const bf16_t* src = qb + row_at(pos, rem, min(r, most)) * DH + 8 * c;
            __builtin_amdgcn_global_load_lds((glb_ptr)src, (lds_ptr)(dst + (wave * NI + j) * 1024), 16, 0, 0);
        }
#pragma unroll
        for (int h = 0; h < HALVES; ++h) L[h] = lb[row_at(pos, rem, min(32 * h + lr, most))];
    };
    if (t0 < t1) issue(t0, smem);
    // the old sums that this lane will add to (lanes 2v of a half: value v of each block)
    const int mykey = 8 * (lr >> 3) + 4 * eta + ((lr >> 1) & 3);
    float old[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
        const int key = k0 + 32 * kb + mykey;
        old[kb] = a.decay != 0.f && nsplit == 1 && key < p ? a.weights[(size_t)un.head * a.ldw + key] : 0.f;
    }
    const float sl2 = a.scale * kLog2e;
    float acc[KB][16];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[kb][v] = 0.f;

    for (int t = t0; t < t1; ++t) {
        char* cur = smem + ((t - t0) & 1) * STAGE;
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();                                     // stage t has arrived, and stage t - 1 is read
        float bias[HALVES];
        bool live[HALVES];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {                   // (a row without a sum counts nothing; NaN stays NaN)
            live[h] = t * kWRows + 32 * h + lr < rows && (fabsf(L[h]) < INFINITY || L[h] != L[h]);
            bias[h] = -L[h] * kLog2e;
        }
        if (t + 1 < t1) issue(t + 1, smem + ((t + 1 - t0) & 1) * STAGE);
        // products of PART halves of the stage in turn, then their exponentials
        constexpr int PART = KB == 2 ? HALVES : 1;
#pragma unroll
        for (int h0 = 0; h0 < HALVES; h0 += PART) {
            floatx16 sc[PART][KB];
            bool all = true;
#pragma unroll
            for (int h = 0; h < PART; ++h) {
                bf16x8 qf[NC];
                const int r = 32 * (h0 + h) + lr;
                all = all && __all(live[h0 + h]);
#pragma unroll
                for (int c = 0; c < NC; ++c)
                    qf[c] = *reinterpret_cast<const bf16x8*>(cur + 16 * (r * CH + (ch(c) ^ swz(r))));
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int v = 0; v < 16; ++v) sc[h][kb][v] = 0.f;
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) sc[h][kb] = mfma32x32x16(kf[kb][c], qf[c], sc[h][kb]);
            }
            if (all) {
#pragma unroll
                for (int h = 0; h < PART; ++h)
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                        for (int v = 0; v < 16; ++v) acc[kb][v] += __builtin_amdgcn_exp2f(fmaf(sc[h][kb][v], sl2, bias[h0 + h]));
            } else {
#pragma unroll
                for (int h = 0; h < PART; ++h)
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                        for (int v = 0; v < 16; ++v)
                            acc[kb][v] += live[h0 + h] ? __builtin_amdgcn_exp2f(fmaf(sc[h][kb][v], sl2, bias[h0 + h])) : 0.f;
            }
        }
    }
    // element v of block kb is key 32 kb + 8 (v / 4) + 4 eta + v % 4
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
        const float x = half_sums(acc[kb], lr);
        const int key = k0 + 32 * kb + mykey;
        if ((lr & 1) == 0 && key < p) {
            if (nsplit > 1) a.part[((size_t)split * a.b * a.Hkv + un.head) * a.P + key] = x;
            else a.weights[(size_t)un.head * a.ldw + key] = fmaf(a.decay, old[kb], x);
        }
    }
}

// Few rows (up to 32 HB): the rows stay in a wave's registers and its keys stream
// through them, a block of 32 ahead of the one at work; no LDS, no barrier.  S = Q K^T,
// so a lane holds 16 rows' scores of one key and adds them by itself.
template <int DH, int HB, bool KV8>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void key_weights_few_kernel(KeyWeightArgs a, int blocks) {
    constexpr int NC = DH / 16, NL = KV8 ? NC / 2 : NC;      // MFMA steps; 16-byte loads of a lane
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane & 31, eta = lane >> 5;
    const WeightUnit un = weight_unit(a, 1, 128 * blocks);   // (a wave takes `blocks` blocks in a row)
    const int g = un.head % a.Hkv, s = un.head / a.Hkv;
    const int p = prefix_len(a.prefix, s, a.P), k0 = (un.kt * 4 + wave) * 32 * blocks, k1 = min(p, k0 + 32 * blocks);
    if (k0 >= k1) return;
    const int GQ = a.Hq / a.Hkv, rows = GQ * a.R;
    auto ch = [&](int c) __attribute__((always_inline)) { return 4 * (c >> 1) + 2 * eta + (c & 1); };   // (as above)
    const char* kb = reinterpret_cast<const char*>(a.k) + ((size_t)s * a.Hkv + g) * a.cap * DH * (KV8 ? 1 : 2);
    float* w = a.weights + (size_t)un.head * a.ldw;
    u32x4 next[NL];
    float old;
    auto fetch = [&](int k) __attribute__((always_inline)) {
        const int key = min(k + lr, p - 1);
#pragma unroll
        for (int c = 0; c < NL; ++c)
            next[c] = KV8 ? *reinterpret_cast<const u32x4*>(kb + (size_t)key * DH + 8 * ch(2 * c))
                          : *reinterpret_cast<const u32x4*>(kb + ((size_t)key * DH + 8 * ch(c)) * 2);
        old = a.decay != 0.f ? w[key] : 0.f;
    };
    fetch(k0);
    // the rows: A operand row lr of block h, and -L of the 16 rows whose scores the lane holds
    bf16x8 qf[HB][NC];
    float bias[HB][16];
    uint32_t live = 0;                                       // bit 16 h + v (a row without a sum counts nothing)
    const size_t base = (size_t)s * a.R * a.Hq + (size_t)g * GQ;
#pragma unroll
    for (int h = 0; h < HB; ++h) {
        const int rho = min(32 * h + lr, rows - 1);
        const bf16_t* q = reinterpret_cast<const bf16_t*>(a.q) + (base + (size_t)(rho / GQ) * a.Hq + rho % GQ) * DH;
#pragma unroll
        for (int c = 0; c < NC; ++c) qf[h][c] = ld_bf16x8(q + 8 * ch(c));
        const float mine = 32 * h + lr < rows ? a.lse[base + (size_t)(rho / GQ) * a.Hq + rho % GQ] : INFINITY;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const float L = __shfl(mine, 8 * (v >> 2) + 4 * eta + (v & 3), 64);
            bias[h][v] = -L * kLog2e;
            if (fabsf(L) < INFINITY || L != L) live |= 1u << (16 * h + v);
        }
    }
    const bool all = __all(live == (HB == 2 ? 0xFFFFFFFFu : 0xFFFFu));
    const float sl2 = a.scale * kLog2e;
    for (int k = k0; k < k1; k += 32) {
        bf16x8 kf[NC];
#pragma unroll
        for (int c = 0; c < NL; ++c) {
            if constexpr (KV8) {
                kf[2 * c] = __builtin_bit_cast(bf16x8, e4m3x8_to_bf16x8_scaled(next[c][0], next[c][1]));
                kf[2 * c + 1] = __builtin_bit_cast(bf16x8, e4m3x8_to_bf16x8_scaled(next[c][2], next[c][3]));
            } else {
                kf[c] = __builtin_bit_cast(bf16x8, next[c]);
            }
        }
        const float was = old;
        if (k + 32 < k1) fetch(k + 32);
        floatx16 sc[HB];
#pragma unroll
        for (int h = 0; h < HB; ++h)
#pragma unroll
            for (int v = 0; v < 16; ++v) sc[h][v] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int h = 0; h < HB; ++h) sc[h] = mfma32x32x16(qf[h][c], kf[c], sc[h]);
        float x = 0.f, y = 0.f;
        if (all) {
#pragma unroll
            for (int h = 0; h < HB; ++h)
#pragma unroll
                for (int v = 0; v < 16; v += 2) {
                    x += __builtin_amdgcn_exp2f(fmaf(sc[h][v], sl2, bias[h][v]));
                    y += __builtin_amdgcn_exp2f(fmaf(sc[h][v + 1], sl2, bias[h][v + 1]));
                }
        } else {
#pragma unroll
            for (int h = 0; h < HB; ++h)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(sc[h][v], sl2, bias[h][v]));
                    x += (live >> (16 * h + v)) & 1u ? e : 0.f;
                }
        }
        x += y;
        x += __shfl_xor(x, 32, 64);
        if (eta == 0 && k + lr < k1) w[k + lr] = fmaf(a.decay, was, x);
    }
}

// The same on v_mfma_f32_16x16x4_f32: a wave takes 32 keys, rows come straight from memory
// where they are used: 64 rows of 4 x 32 heads of 128, up to 2048 keys 46 us, three times what
// the keys' bytes, or the products, take at full rate.
template <int DH>
__global__ __launch_bounds__(256) void key_weights_f32_kernel(KeyWeightArgs a, int nsplit) {
    constexpr int NC = DH / 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane & 15, q4 = lane >> 4;
    const WeightUnit un = weight_unit(a, nsplit, 128);
    const int g = un.head % a.Hkv, s = un.head / a.Hkv, kt = un.kt, split = un.split;
    const int p = prefix_len(a.prefix, s, a.P), k0 = (kt * 4 + wave) * 32;
    if (k0 >= p) return;
    const int GQ = a.Hq / a.Hkv, rows = GQ * a.R, ntile = (rows + 15) / 16;
    const int t0 = (int)((long long)ntile * split / nsplit), t1 = (int)((long long)ntile * (split + 1) / nsplit);
    const float* qb = reinterpret_cast<const float*>(a.q) + ((size_t)s * a.R * a.Hq + (size_t)g * GQ) * DH;
    const float* lb = a.lse + (size_t)s * a.R * a.Hq + (size_t)g * GQ;
    floatx4 kf[2][NC];
    float acc[2][4] = {};
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int c = 0; c < NC; ++c)
            kf[kb][c] = ld_f4(reinterpret_cast<const float*>(a.k) +
                              (((size_t)s * a.Hkv + g) * a.cap + min(k0 + 16 * kb + lr, p - 1)) * DH + 16 * c + 4 * q4);
    for (int t = t0; t < t1; ++t) {
        const int rho = t * 16 + lr, rc = min(rho, rows - 1);
        const size_t at = (size_t)(rc / GQ) * a.Hq + rc % GQ;
        const float L = rho < rows ? lb[at] : INFINITY;
        const bool live = fabsf(L) < INFINITY || L != L;
        floatx4 qf[NC], sc[2];
#pragma unroll
        for (int c = 0; c < NC; ++c) qf[c] = ld_f4(qb + at * DH + 16 * c + 4 * q4);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            sc[kb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[kb] = mfma16x16x4f(kf[kb][c][e], qf[c][e], sc[kb]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                acc[kb][e] += live ? __builtin_amdgcn_exp2f((fmaf(sc[kb][e], a.scale, -L)) * kLog2e) : 0.f;
        }
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x = acc[kb][e];
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
            const int key = k0 + 16 * kb + 4 * q4 + e;
            if (lr == 0 && key < p) {
                if (nsplit > 1) a.part[((size_t)split * a.b * a.Hkv + un.head) * a.P + key] = x;
                else add_weight(a, un.head, key, x);
            }
        }
}

// Partial sums of a row split, added in order.
__global__ __launch_bounds__(256) void key_weights_sum_kernel(KeyWeightArgs a, int nsplit) {
    const int blocks = (a.P + 255) / 256, head = blockIdx.x / blocks;
    const int key = blockIdx.x % blocks * 256 + threadIdx.x;
    if (key >= prefix_len(a.prefix, head / a.Hkv, a.P)) return;
    float x = 0.f;
#pragma unroll 4
    for (int i = 0; i < nsplit; ++i) x += a.part[((size_t)i * a.b * a.Hkv + head) * a.P + key];
    add_weight(a, head, key, x);
}

struct WeightCfg {
    int few;          // rows in registers: blocks of 32 rows, else 0
    int kb, ktiles, ns;
};

WeightCfg weight_cfg(int dtype, int b, int R, int Hq, int Hkv, int P) {
    WeightCfg c{};
    const long rows = (long)R * (Hq / Hkv), heads = (long)b * Hkv;
    // Few rows stay in registers where the keys are enough for 8 waves a CU (kb: blocks of
    // 32 that a wave takes in a row): 64 rows of 16 x 32 heads, FP8, up to 1664 keys 22 us
    // (rows in LDS: 28), 8 rows of 8 x 32 heads over 4096 keys 44 (56); 64 rows of 32 heads
    // over 609 keys 6.3 (5.3).
    const long blocks = heads * ((P + 31) / 32);
    if (dtype != DARD_DTYPE_F32 && rows <= 64 && blocks >= 2048) {
        c.few = rows > 32 ? 2 : 1;
        c.kb = (int)std::min<long>(16, blocks / 2048);
        c.ktiles = (P + 128 * c.kb - 1) / (128 * c.kb);
        c.ns = 1;
        return c;
    }
    c.kb = dtype == DARD_DTYPE_F32 || rows < 512 || heads * ((P + 255) / 256) < 256 ? 1 : 2;
    c.ktiles = (P + 128 * c.kb - 1) / (128 * c.kb);
    const long wgs = heads * c.ktiles, tiles = (rows + kWRows - 1) / kWRows;
    c.ns = (int)std::max<long>(1, std::min<long>(512 / wgs, tiles / 4));
    return c;
}

// ---------------------------------------------------------------- selection
// The m = min(n, length) keys of a (sequence, KV head) row of sums that rank
// highest: protected keys first, then by sum, ties to the lowest index.  Sums
// map to unsigned integers of the same order (NaN below minus infinity, -0 as 0,
// protected keys above all), and the rank's threshold is found digit by digit
// from histograms in LDS.  One workgroup a row; each of its waves owns a run of
// consecutive keys, counts what it keeps, and writes its indices behind those of
// the waves before it.  Bound by the chain of barriers and histogram counts, not by
// bytes: 8 rows of 609 sums 5.7 us, 512 of 1664 8.8, 4 of 131072 (several workgroups a
// row) 32 in four launches.
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;

__device__ __forceinline__ uint32_t sum_rank(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
    return (u >> 31) ? ~u : u | 0x80000000u;                 // -inf: 0x007FFFFF; +inf: 0xFF800000
}

// HELD: the row's sums fit the registers (HELD keys a thread) and are read once; 0:
// every pass reads them again, 16 keys a thread in flight.
// A digit's bin that is taken whole ends the search.
// BITS: of a digit; short rows take four of 8 bits in workgroups of 256 threads, whose
// barriers are quick, others three of 11 in 1024.
template <int THREADS, int HELD, int BITS>
__global__ __launch_bounds__(THREADS) void kv_select_kernel(KvSelectArgs a) {
    // histogram copies by lane: equal sums in neighbouring lanes would queue at one counter
    constexpr int COPIES = 4, WAVES = THREADS / 64, BINS = 1 << BITS, BPT = BINS / THREADS, DIGITS = (32 + BITS - 1) / BITS;
    static_assert(BPT == 1 || BPT == 2, "a bin or two a thread");
    __shared__ uint32_t hist[COPIES][BINS];
    __shared__ uint32_t wsum[WAVES], wtie[WAVES];
    __shared__ uint32_t found[3];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int s = blockIdx.x / a.Hkv;
    const int p = prefix_len(a.prefix, s, a.P), m = min(a.n, p);
    const float* w = a.weights + (size_t)blockIdx.x * a.ldw;
    int32_t* keep = a.keep + (size_t)blockIdx.x * a.n;
    if (a.kept && blockIdx.x % a.Hkv == 0 && tid == 0) a.kept[s] = m;
    for (int i = m + tid; i < a.n; i += THREADS) keep[i] = -1;
    if (m == p) {                                            // nothing to leave out
        for (int i = tid; i < m; i += THREADS) keep[i] = i;
        return;
    }
    // a wave's keys: a run of whole 256s, four neighbours a lane
    const int per = ((p + WAVES - 1) / WAVES + 255) / 256 * 256, j0 = wave * per, j1 = min(p, j0 + per);
    auto fetch = [&](int j) __attribute__((always_inline)) {
        floatx4 x = {0.f, 0.f, 0.f, 0.f};
        if (j + 4 <= p) x = ld_f4(w + j);
        else if (j < p)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = w[min(j + e, p - 1)];
        return x;
    };
    auto rank = [&](float x, int j) __attribute__((always_inline)) {
        return j < a.first || j >= p - a.last ? 0xFFFFFFFFu : sum_rank(x);
    };
    floatx4 held[HELD ? HELD / 4 : 1];
    if constexpr (HELD > 0) {
#pragma unroll
        for (int i = 0; i < HELD / 4; ++i) held[i] = fetch(j0 + 256 * i + 4 * lane);
    }
    // f(ranks of four keys, index of the first) over the wave's run, in order
    auto run = [&](auto f) __attribute__((always_inline)) {
        auto four = [&](floatx4 x, int j) __attribute__((always_inline)) {
            uint32_t u[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = rank(x[e], j + e);
            f(u, j);
        };
        if constexpr (HELD > 0) {
#pragma unroll
            for (int i = 0; i < HELD / 4; ++i)
                if (j0 + 256 * i < j1) four(held[i], j0 + 256 * i + 4 * lane);
        } else {
            for (int j = j0; j < j1; j += 1024) {
                floatx4 x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = fetch(j + 256 * i + 4 * lane);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (j + 256 * i < j1) four(x[i], j + 256 * i + 4 * lane);
            }
        }
    };
    // threshold T: fewer than m keys rank above it, m or more at or above it
    uint32_t T = 0, mask = 0;
    int need = m;                                            // keys to take among those that agree with T under mask
#pragma unroll
    for (int d = 0; d < DIGITS; ++d) {
        const int shift = d + 1 < DIGITS ? 32 - BITS * (d + 1) : 0, bits = d + 1 < DIGITS ? BITS : 32 - BITS * d;
#pragma unroll
        for (int i = 0; i < COPIES * BINS / THREADS; ++i) (&hist[0][0])[i * THREADS + tid] = 0;
        __syncthreads();
        run([&](const uint32_t (&u)[4], int j) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (j + e < j1 && (u[e] & mask) == T) atomicAdd(&hist[lane % COPIES][(u[e] >> shift) & ((1u << bits) - 1)], 1u);
        });
        __syncthreads();
        // the bin in which the count from the top passes need (integer counts: order plays no part)
        uint32_t c[BPT], sum = 0;                            // this thread's bins, from the top
#pragma unroll
        for (int i = 0; i < BPT; ++i) {
            c[i] = 0;
#pragma unroll
            for (int k = 0; k < COPIES; ++k) c[i] += hist[k][BINS - 1 - BPT * tid - i];
            sum += c[i];
        }
        const uint32_t mine = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t below = __shfl_up(sum, o, 64);
            if (lane >= o) sum += below;
        }
        if (lane == 63) wsum[wave] = sum;
        __syncthreads();
        uint32_t before = sum - mine;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) before += i < wave ? wsum[i] : 0u;
        const uint32_t want = (uint32_t)need;
#pragma unroll
        for (int i = 0; i < BPT; ++i) {
            if (before < want && before + c[i] >= want) {
                found[0] = BINS - 1 - BPT * tid - i;
                found[1] = before;
                found[2] = before + c[i] == want;
            }
            before += c[i];
        }
        __syncthreads();
        T |= found[0] << shift;
        mask |= ((1u << bits) - 1) << shift;
        need -= (int)found[1];
        if (found[2]) {                                      // the whole bin: all above T - 1, none that equals it
            --T;
            need = 0;
            break;
        }
    }
    // keys above T, and the first `need` of those that equal it, in index order
    uint32_t above = 0, ties = 0;
    run([&](const uint32_t (&u)[4], int j) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            above += j + e < j1 && u[e] > T;
            ties += j + e < j1 && u[e] == T;
        }
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        above += __shfl_xor(above, o, 64);
        ties += __shfl_xor(ties, o, 64);
    }
    if (lane == 0) { wsum[wave] = above; wtie[wave] = ties; }
    __syncthreads();
    uint32_t pos = 0, tie = 0;                               // keys above T, and ties, before this wave's run
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        pos += i < wave ? wsum[i] : 0u;
        tie += i < wave ? wtie[i] : 0u;
    }
    const uint64_t lower = (1ull << lane) - 1;
    run([&](const uint32_t (&u)[4], int j) __attribute__((always_inline)) {
        uint32_t up = pos, eq = tie;                         // before this lane's four keys
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint64_t ba = __ballot(j + e < j1 && u[e] > T), bt = __ballot(j + e < j1 && u[e] == T);
            up += __builtin_popcountll(ba & lower);
            eq += __builtin_popcountll(bt & lower);
            pos += __builtin_popcountll(ba);
            tie += __builtin_popcountll(bt);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (j + e >= j1) continue;
            if (u[e] > T || (u[e] == T && eq < (uint32_t)need)) keep[up + min(eq, (uint32_t)need)] = j + e;
            up += u[e] > T;
            eq += u[e] == T;
        }
    });
}

// Short rows: one wave a row, no LDS and no barrier.  The threshold is found bit by bit
// from the top, with a compare and a scalar count for every 64 keys, and the search ends
// at the first bit that leaves exactly m keys at or above it.  (4096 rows of 500 sums 10
// us, 8 of 300 5; a workgroup of 256 threads a row 16 and 5.5.  With 16 keys a lane the
// counts take longer than histograms: 8 rows of 609 7.7 and 5.7.)
constexpr int kWaveKeys = 8;                                 // of a lane

__global__ __launch_bounds__(64) void kv_select_wave_kernel(KvSelectArgs a) {
    constexpr int HELD = kWaveKeys;
    const int lane = threadIdx.x, s = blockIdx.x / a.Hkv;
    const int p = prefix_len(a.prefix, s, a.P), m = min(a.n, p);
    const float* w = a.weights + (size_t)blockIdx.x * a.ldw;
    int32_t* keep = a.keep + (size_t)blockIdx.x * a.n;
    if (a.kept && blockIdx.x % a.Hkv == 0 && lane == 0) a.kept[s] = m;
    for (int i = m + lane; i < a.n; i += 64) keep[i] = -1;
    if (m == p) {                                            // nothing to leave out
        for (int i = lane; i < m; i += 64) keep[i] = i;
        return;
    }
    floatx4 x[HELD / 4];
#pragma unroll
    for (int i = 0; i < HELD / 4; ++i) {
        const int j = 256 * i + 4 * lane;
        x[i] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (j + 4 <= p) x[i] = ld_f4(w + j);
        else if (j < p)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][e] = w[min(j + e, p - 1)];
    }
    uint32_t u[HELD];                                        // (0 past the last key: under every threshold but 0)
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int j = 256 * (i >> 2) + 4 * lane + (i & 3);
        u[i] = j >= p ? 0u : j < a.first || j >= p - a.last ? 0xFFFFFFFFu : sum_rank(x[i >> 2][i & 3]);
    }
    // T: fewer than m keys rank above it, m or more at or above it
    auto count = [&](uint32_t t) __attribute__((always_inline)) {
        uint32_t c = 0;
#pragma unroll
        for (int i = 0; i < HELD; ++i) c += __builtin_popcountll(__ballot(u[i] >= t));
        return c;
    };
    uint32_t T = 0, ties = 0;                                // ties: of the keys that equal T, how many to take
    bool exact = false;
    for (uint32_t bit = 0x80000000u; bit && !exact; bit >>= 1) {
        const uint32_t c = count(T | bit);
        if (c >= (uint32_t)m) T |= bit;
        exact = c == (uint32_t)m;
    }
    if (exact) --T;                                          // all above T - 1, none of those that equal it
    else ties = m - (T == 0xFFFFFFFFu ? 0u : count(T + 1));
    uint32_t pos = 0, tie = 0;                               // keys above T, and ties, so far
    const uint64_t lower = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < HELD; i += 4) {
        const int j = 256 * (i >> 2) + 4 * lane;
        uint32_t up = pos, eq = tie;                         // before this lane's four keys
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint64_t ba = __ballot(u[i + e] > T), bt = __ballot(j + e < p && u[i + e] == T);
            up += __builtin_popcountll(ba & lower);
            eq += __builtin_popcountll(bt & lower);
            pos += __builtin_popcountll(ba);
            tie += __builtin_popcountll(bt);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x = u[i + e];
            if (j + e >= p) continue;
            if (x > T || (x == T && eq < ties)) keep[up + min(eq, ties)] = j + e;
            up += x > T;
            eq += x == T;
        }
    }
}

// Long rows of few heads: every digit's histogram, and the indices, in a launch of
// their own with a workgroup per chunk of kChunk keys.  A workgroup adds the chunks'
// histograms of the digit before to find the threshold's bin, as each of the others
// does (nothing has to be initialised, or to meet), and the first one leaves it for
// the launches to come; so does each its own chunk's count above the threshold so far.
// From those counts follows where its indices go.
constexpr int kChunkKeys = 16;                               // keys a thread
constexpr int kChunk = kSelThreads * kChunkKeys, kBins = 2048;

template <int digit>
__global__ __launch_bounds__(kSelThreads) void kv_select_long_kernel(KvSelectArgs a, int chunks) {
    constexpr int COPIES = 4;                                // (by lane, as in kv_select_kernel)
    __shared__ uint32_t hist[COPIES][kBins];
    __shared__ uint32_t wsum[kSelWaves], wtie[kSelWaves];
    __shared__ uint32_t found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.x / chunks, chunk = blockIdx.x % chunks, s = row / a.Hkv;
    const int p = prefix_len(a.prefix, s, a.P), m = min(a.n, p);
    constexpr bool last = digit == 3;
    int32_t* keep = a.keep + (size_t)row * a.n;
    const int c0 = chunk * kChunk;
    if (last) {
        if (a.kept && row % a.Hkv == 0 && chunk == 0 && tid == 0) a.kept[s] = m;
        for (int i = max(m, c0) + tid; i < min(a.n, chunk + 1 == chunks ? a.n : c0 + kChunk); i += kSelThreads) keep[i] = -1;
        if (m == p)
            for (int i = c0 + tid; i < min(m, c0 + kChunk); i += kSelThreads) keep[i] = i;
    }
    if (m == p || c0 >= p) return;
    // this wave's keys: whole 256s in a row, four neighbours a lane
    const int j0 = c0 + wave * 64 * kChunkKeys;
    uint32_t u[kChunkKeys];
    bool in[kChunkKeys];
    {
        const float* w = a.weights + (size_t)row * a.ldw;
        floatx4 x[kChunkKeys / 4];
#pragma unroll
        for (int i = 0; i < kChunkKeys / 4; ++i) {
            const int j = j0 + 256 * i + 4 * lane;
            x[i] = floatx4{0.f, 0.f, 0.f, 0.f};
            if (j + 4 <= p) x[i] = ld_f4(w + j);
            else if (j < p)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[i][e] = w[min(j + e, p - 1)];
        }
#pragma unroll
        for (int i = 0; i < kChunkKeys; ++i) {
            const int j = j0 + 256 * (i >> 2) + 4 * lane + (i & 3);
            in[i] = j < p;
            u[i] = j < a.first || j >= p - a.last ? 0xFFFFFFFFu : sum_rank(x[i >> 2][i & 3]);
        }
    }
    const int rows = gridDim.x / chunks;
    uint32_t* state = a.ws + (size_t)3 * gridDim.x * kBins;  // [digit][row]: bin, keys above it; then [digit][row][chunk] counts
    uint32_t* counts = state + (size_t)6 * rows;
    uint32_t T = 0, mask = 0, pos = 0, tie = 0;              // pos, tie: keys above T, and ties, of the chunks before this one
    int need = m;
    // what the launches before left, on its way together
    uint2 left[2] = {};
    uint32_t before0 = 0;
#pragma unroll
    for (int d = 0; d + 1 < digit; ++d) {
        left[d] = reinterpret_cast<const uint2*>(state)[(size_t)d * rows + row];
        if (last)
            for (int c = lane; c < chunk; c += 64) before0 += counts[((size_t)d * rows + row) * chunks + c];
    }
#pragma unroll
    for (int d = 0; d < digit; ++d) {
        const int shift = d == 0 ? 21 : d == 1 ? 10 : 0, bits = d == 2 ? 10 : 11;
        uint32_t bin, over;
        if (d + 1 < digit) {
            bin = left[d].x;
            over = left[d].y;
        } else {
            // this thread's two bins, from the top; their counts in this chunk and in those before it
            const uint32_t* h = a.ws + ((size_t)d * gridDim.x + (size_t)row * chunks) * kBins + 2046 - 2 * tid;
            uint32_t n0 = 0, n1 = 0, b0 = 0, b1 = 0, o0 = 0, o1 = 0;
#pragma unroll 4
            for (int c = 0; c * kChunk < p; ++c) {
                const uint2 v = *reinterpret_cast<const uint2*>(h + (size_t)c * kBins);
                n0 += v.y;
                n1 += v.x;
                b0 += c < chunk ? v.y : 0u;
                b1 += c < chunk ? v.x : 0u;
                o0 += c == chunk ? v.y : 0u;
                o1 += c == chunk ? v.x : 0u;
            }
            uint32_t sum = n0 + n1;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const uint32_t below = __shfl_up(sum, o, 64);
                if (lane >= o) sum += below;
            }
            if (lane == 63) wsum[wave] = sum;
            __syncthreads();
            uint32_t before = sum - n0 - n1;
#pragma unroll
            for (int i = 0; i < kSelWaves; ++i) before += i < wave ? wsum[i] : 0u;
            const uint32_t want = (uint32_t)need;
            if (before < want && before + n0 >= want) { found[0] = 2047 - 2 * tid; found[1] = before; }
            if (before + n0 < want && before + n0 + n1 >= want) { found[0] = 2046 - 2 * tid; found[1] = before + n0; }
            __syncthreads();
            bin = found[0];
            over = found[1];
            const uint32_t top = 2047 - 2 * tid;
            // (not the last launch: this chunk's keys above the bin; the last: those of the chunks before, and ties)
            uint32_t up = last ? (top > bin ? b0 : 0u) + (top - 1 > bin ? b1 : 0u) : (top > bin ? o0 : 0u) + (top - 1 > bin ? o1 : 0u);
            uint32_t eq = (top == bin ? b0 : 0u) + (top - 1 == bin ? b1 : 0u);
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) {
                up += __shfl_xor(up, o, 64);
                eq += __shfl_xor(eq, o, 64);
            }
            if (lane == 0) { wsum[wave] = up; wtie[wave] = eq; }   // (every wave has read found: the sync below)
            __syncthreads();
            up = eq = 0;
#pragma unroll
            for (int i = 0; i < kSelWaves; ++i) { up += wsum[i]; eq += wtie[i]; }
            if (last) {
#pragma unroll
                for (int o = 32; o > 0; o >>= 1) before0 += __shfl_xor(before0, o, 64);
                pos = up + before0;
                tie = eq;
            } else if (tid == 0) {
                counts[((size_t)d * rows + row) * chunks + chunk] = up;
                if (chunk == 0) reinterpret_cast<uint2*>(state)[(size_t)d * rows + row] = make_uint2(bin, over);
            }
        }
        T |= bin << shift;
        mask |= ((1u << bits) - 1) << shift;
        need -= (int)over;
    }
    if (!last) {
#pragma unroll
        for (int i = 0; i < COPIES * kBins / kSelThreads; ++i) (&hist[0][0])[i * kSelThreads + tid] = 0;
        __syncthreads();
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
#pragma unroll
        for (int i = 0; i < kChunkKeys; ++i)
            if (in[i] && (u[i] & mask) == T) atomicAdd(&hist[lane % COPIES][(u[i] >> shift) & ((1u << bits) - 1)], 1u);
        __syncthreads();
        uint32_t* h = a.ws + ((size_t)digit * gridDim.x + blockIdx.x) * kBins;
#pragma unroll
        for (int i = 0; i < kBins; i += kSelThreads) h[i + tid] = hist[0][i + tid] + hist[1][i + tid] + hist[2][i + tid] + hist[3][i + tid];
        return;
    }
    // this chunk's waves before this one (counts of a wave are under 2^16: two in a register)
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < kChunkKeys; ++i) mine += in[i] ? (u[i] > T ? 1u : 0u) + (u[i] == T ? 1u << 16 : 0u) : 0u;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o, 64);
    __syncthreads();
    if (lane == 0) { wsum[wave] = mine & 0xFFFFu; wtie[wave] = mine >> 16; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSelWaves; ++i) {
        pos += i < wave ? wsum[i] : 0u;
        tie += i < wave ? wtie[i] : 0u;
    }
    const uint64_t lower = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < kChunkKeys; i += 4) {
        uint32_t up = pos, at = tie;                         // before this lane's four keys
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint64_t ba = __ballot(in[i + e] && u[i + e] > T), bt = __ballot(in[i + e] && u[i + e] == T);
            up += __builtin_popcountll(ba & lower);
            at += __builtin_popcountll(bt & lower);
            pos += __builtin_popcountll(ba);
            tie += __builtin_popcountll(bt);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x = u[i + e];
            if (!in[i + e]) continue;
            if (x > T || (x == T && at < (uint32_t)need)) keep[up + min(at, (uint32_t)need)] = j0 + 256 * (i >> 2) + 4 * lane + e;
            up += x > T;
            at += x == T;
        }
    }
}

// ---------------------------------------------------------------- compaction
// Key j of a (sequence, KV head) becomes key keep[j], in place.  keep ascends, so
// keep[j] >= j: chunk by chunk a workgroup reads the sources of a run of places,
// then writes that run, which no later chunk reads.  A workgroup owns whole
// columns (a run of a key's bytes, or rows of the dims-major V), so the order of
// reads and writes is its own affair.  Bound by memory: kept keys are read and written,
// and of V whole lines are read for the keys of them that are kept.  Scattered sources, from
// memory: 16 sequences x 32 heads of 128, up to 1664 -> 1024 keys 52 us; 4 heads, 131072 -> 32768
// keys 50 and 12 us, 235 MB at 3.7 TB/s.  16 x 32 heads, 1664 -> 1024 keys each: fp32 238 us, bf16 121,
// FP8 82 (V is loaded byte by byte, four loads for a word that is stored), 1.1, 1.1 and 1.5 times
// what the kept keys alone take at a copy's rate.
// Sources ascend, so keep[j] = j for a leading run of places and for no other: how many
// whole chunks of it need no move (64 probes a step).
__device__ __forceinline__ int chunks_in_place(const int32_t* keep, int m, int chunk) {
    int n = 0;
    for (;;) {
        const long long end = min((long long)(n + (int)(threadIdx.x & 63) + 1) * chunk, (long long)m);
        const uint64_t moved = __ballot(keep[end - 1] != (int)end - 1);
        if (moved) return n + __builtin_ctzll(moved);
        n += 64;
        if ((long long)n * chunk >= m) return n;
    }
}

// What is written before stays before.
__device__ __forceinline__ void in_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Every source of a chunk that any wave has asked for is in registers: only then is the
// chunk written.  (All loads and stores are waited for, not a count of the newer ones: that
// would rest on the order and the number of instructions that the compiler makes of them.  The
// indices of the next chunk, which are newer than its sources, are waited for here in any case.)
__device__ __forceinline__ void sources_read() {
    in_order();
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    wg_barrier();
}

// A workgroup owns SEG bytes of every key; a thread moves 16 bytes at a time, the
// next chunk's loads under way while a chunk is written.  (Places past the last one
// read its source again: loads without branches go out together.)
// NEAR: only the places whose source lies among the m places (a leading run, since
// sources ascend); the others depend on no order (move_far_keys).
template <int THREADS, int SEG, bool NEAR, int U = 8>
__device__ __forceinline__ void move_keys(char* k, int row_bytes, const int32_t* keep, int m, int P) {
    constexpr int LPR = SEG / 16, STEP = THREADS / LPR;      // lanes a key, keys a pass (U of them a chunk)
    const int tid = threadIdx.x, key = tid / LPR, at = tid % LPR * 16;
    if (m < 1) return;
    u32x4 x[U];
    int src[U];
    auto indices = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) src[u] = min(max(keep[min(j0 + u * STEP + key, m - 1)], 0), P - 1);
    };
    auto load = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = *reinterpret_cast<const u32x4e*>(k + (size_t)src[u] * row_bytes + at);
    };
    indices(0);
    const int at0 = chunks_in_place(keep, m, U * STEP);
    if ((long long)at0 * U * STEP >= m) return;
    const int first = at0 * U * STEP;
    if (first) indices(first);
    load();
    in_order();
    indices(first + U * STEP);
    for (int j0 = first; j0 < m; j0 += U * STEP) {
        if (NEAR && keep[j0] >= m) break;
        u32x4 y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) y[u] = x[u];
        sources_read();
        if (j0 + U * STEP < m) load();
        indices(j0 + 2 * U * STEP);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u * STEP + key;
            if (j < m && (!NEAR || keep[j] < m)) *reinterpret_cast<u32x4e*>(k + (size_t)j * row_bytes + at) = y[u];
        }
    }
}

// The places whose source lies behind the m places: nothing that is written is read
// any more once the others have moved, so every workgroup takes places of its own.
template <int THREADS, int U>
__device__ __forceinline__ void move_far_keys(char* k, int row_bytes, const int32_t* keep, int m, int P, int j0) {
    const int lpr = row_bytes / 16, step = THREADS / lpr, at = threadIdx.x % lpr * 16;
    u32x4 x[U];
    bool far[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int j = j0 + u * step + (int)threadIdx.x / lpr, src = keep[min(j, m - 1)];
        far[u] = j < m && src >= m;
        x[u] = *reinterpret_cast<const u32x4e*>(k + (size_t)min(max(src, 0), P - 1) * row_bytes + at);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (far[u]) *reinterpret_cast<u32x4e*>(k + (size_t)(j0 + u * step + threadIdx.x / lpr) * row_bytes + at) = x[u];
}

// A workgroup owns ROWS rows of `cap` elements; a thread takes the elements of 4
// bytes of a row at a time: their sources lie close together (the share of keys
// that is kept apart), so single loads reach whole lines between a wave's lanes.
template <typename T> struct Word;   // 4 bytes at an element's alignment, over elements that are loaded as T
template <> struct Word<float> { typedef uint32_t type __attribute__((may_alias)); };
template <> struct Word<uint16_t> { typedef uint32_t type __attribute__((aligned(2), may_alias)); };
template <> struct Word<uint8_t> { typedef uint32_t type __attribute__((aligned(1), may_alias)); };

template <typename T, int THREADS, int ROWS, int E>
__device__ __forceinline__ void move_values(T* v, int cap, const int32_t* keep, int m, int P) {
    constexpr int SU = 4 / sizeof(T), CHUNK = THREADS * SU * E;
    const int tid = threadIdx.x;
    if (m < 1) return;
    T x[ROWS][E][SU];
    int src[E][SU];
    auto indices = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int i = 0; i < SU; ++i) src[e][i] = min(max(keep[min(j0 + (e * THREADS + tid) * SU + i, m - 1)], 0), P - 1);
    };
    auto load = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int i = 0; i < SU; ++i)
#pragma unroll
                for (int d = 0; d < ROWS; ++d) x[d][e][i] = v[(size_t)d * cap + src[e][i]];
    };
    indices(0);
    const int at0 = chunks_in_place(keep, m, CHUNK);
    if ((long long)at0 * CHUNK >= m) return;
    const int first = at0 * CHUNK;
    if (first) indices(first);
    load();
    in_order();
    indices(first + CHUNK);
    for (int j0 = first; j0 < m; j0 += CHUNK) {
        uint32_t y[ROWS][E];
#pragma unroll
        for (int d = 0; d < ROWS; ++d)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if constexpr (SU == 1) {
                    y[d][e] = __float_as_uint(x[d][e][0]);
                } else {
                    y[d][e] = 0;
#pragma unroll
                    for (int i = 0; i < SU; ++i) y[d][e] |= (uint32_t)x[d][e][i] << (8 * (int)sizeof(T) * i);
                }
            }
        sources_read();
        if (j0 + CHUNK < m) load();
        indices(j0 + 2 * CHUNK);
#pragma unroll
        for (int d = 0; d < ROWS; ++d)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int j = j0 + (e * THREADS + tid) * SU;
                T* to = v + (size_t)d * cap + j;
                if (j + SU <= m) {
                    *reinterpret_cast<typename Word<T>::type*>(to) = y[d][e];
                } else {
                    if constexpr (SU > 1) {
#pragma unroll
                        for (int i = 0; i < SU; ++i)
                            if (j + i < m) to[i] = (T)(y[d][e] >> (8 * (int)sizeof(T) * i));
                    }
                }
            }
    }
}

// Grid: the parts of every (sequence, KV head), dealt to the XCDs like the key weights'
// units, so that segments of one line meet in one L2: segments of K's rows, groups of
// V's rows, then (with sums) one part for them.
template <typename T, int DH, int THREADS, int SEG, int ROWS, int E, bool NEAR>
__global__ __launch_bounds__(THREADS) void kv_compact_kernel(KvCompactArgs a) {
    constexpr int KP = DH * (int)sizeof(T) / SEG, VP = DH / ROWS;
    const int parts = KP + VP + (a.weights ? 1 : 0), heads = a.b * a.Hkv, per = heads >> 3;
    const int total = gridDim.x, xcd = blockIdx.x & 7, bid = xcd * (total >> 3) + min(xcd, total & 7) + (blockIdx.x >> 3);
    const int slot = bid / parts, head = heads & 7 ? slot : slot % per * 8 + slot / per, s = head / a.Hkv;
    const int p = prefix_len(a.prefix, s, a.P);
    const int m = min(a.kept ? max(a.kept[s], 0) : a.n, min(a.n, p));
    const int32_t* keep = a.keep + (size_t)head * a.n;
    const size_t base = (size_t)head * a.cap * DH;
    int part = bid % parts;
    if (part < KP) {
        move_keys<THREADS, SEG, NEAR>(reinterpret_cast<char*>(a.k) + base * sizeof(T) + part * SEG, DH * sizeof(T), keep, m, p);
        return;
    }
    part -= KP;
    if (part < VP) {
        move_values<T, THREADS, ROWS, E>(reinterpret_cast<T*>(a.v) + base + (size_t)part * ROWS * a.cap, a.cap, keep, m, p);
        return;
    }
    float* w = a.weights + (size_t)head * a.ldw;
    move_values<float, THREADS, 1, THREADS == 1024 ? 32 : 4>(w, 0, keep, m, p);   // (one workgroup a head: many at a time)
    __syncthreads();
    for (int j = m + 4 * (int)threadIdx.x; j < p; j += 4 * THREADS) {            // freed places start from nothing
        if (j + 4 <= p) st_f4(w + j, floatx4{0.f, 0.f, 0.f, 0.f});
        else
            for (int e = j; e < p; ++e) w[e] = 0.f;
    }
}

constexpr int kFarThreads = 256, kFarPasses = 4;

template <typename T, int DH>
__global__ __launch_bounds__(kFarThreads) void kv_compact_far_kernel(KvCompactArgs a, int blocks) {
    constexpr int ROW = DH * (int)sizeof(T);
    const int head = blockIdx.x / blocks, s = head / a.Hkv, p = prefix_len(a.prefix, s, a.P);
    const int m = min(a.kept ? max(a.kept[s], 0) : a.n, min(a.n, p)), j0 = blockIdx.x % blocks * (kFarThreads / (ROW / 16) * kFarPasses);
    if (j0 >= m) return;
    move_far_keys<kFarThreads, kFarPasses>(reinterpret_cast<char*>(a.k) + (size_t)head * a.cap * ROW, ROW, a.keep + (size_t)head * a.n, m, p, j0);
}

}  // namespace

size_t key_weights_partial_floats(int dtype, int b, int R, int Hq, int Hkv, int P) {
    const WeightCfg c = weight_cfg(dtype, b, R, Hq, Hkv, P);
    return c.ns <= 1 ? 0 : (size_t)c.ns * b * Hkv * P;
}

hipError_t launch_key_weights(int dtype, const KeyWeightArgs& a, hipStream_t s) {
    const WeightCfg c = weight_cfg(dtype, a.b, a.R, a.Hq, a.Hkv, a.P);
    const dim3 grid((unsigned)((long)a.b * a.Hkv * c.ktiles * c.ns));
    void (*k)(KeyWeightArgs, int);
    if (c.few) {
        const bool kv8 = dtype == DARD_DTYPE_BF16_KV_FP8, two = c.few == 2;
        if (a.dh == 128) k = kv8 ? (two ? key_weights_few_kernel<128, 2, true> : key_weights_few_kernel<128, 1, true>)
                                 : (two ? key_weights_few_kernel<128, 2, false> : key_weights_few_kernel<128, 1, false>);
        else k = kv8 ? (two ? key_weights_few_kernel<64, 2, true> : key_weights_few_kernel<64, 1, true>)
                     : (two ? key_weights_few_kernel<64, 2, false> : key_weights_few_kernel<64, 1, false>);
        launch(k, dim3((unsigned)((long)a.b * a.Hkv * c.ktiles)), dim3(256), 0, s, a, c.kb);
        return hipGetLastError();
    }
    if (dtype == DARD_DTYPE_F32) k = a.dh == 128 ? key_weights_f32_kernel<128> : key_weights_f32_kernel<64>;
    else if (dtype == DARD_DTYPE_BF16_KV_FP8)
        k = a.dh == 128 ? (c.kb == 2 ? key_weights_kernel<128, 2, true> : key_weights_kernel<128, 1, true>)
                        : (c.kb == 2 ? key_weights_kernel<64, 2, true> : key_weights_kernel<64, 1, true>);
    else
        k = a.dh == 128 ? (c.kb == 2 ? key_weights_kernel<128, 2, false> : key_weights_kernel<128, 1, false>)
                        : (c.kb == 2 ? key_weights_kernel<64, 2, false> : key_weights_kernel<64, 1, false>);
    launch(k, grid, dim3(256), 0, s, a, c.ns);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || c.ns == 1) return e;
    launch(key_weights_sum_kernel, dim3((unsigned)((long)a.b * a.Hkv * ((a.P + 255) / 256))), dim3(256), 0, s, a, c.ns);
    return hipGetLastError();
}

// Chunks of a row where it is long and the rows alone do not fill the chip; else 1.
static int select_chunks(int b, int Hkv, int P) {
    return P > kChunk && (long)b * Hkv <= 128 ? (P - 1) / kChunk + 1 : 1;
}

size_t kv_select_workspace(int b, int Hkv, int P) {
    const int chunks = select_chunks(b, Hkv, P);
    return chunks > 1 ? ((size_t)3 * b * Hkv * chunks * kBins + (size_t)b * Hkv * (6 + 2 * chunks)) * 4 : 0;
}

hipError_t launch_kv_select(const KvSelectArgs& a, hipStream_t s) {
    const int chunks = select_chunks(a.b, a.Hkv, a.P);
    if (chunks > 1) {
        void (*const digits[])(KvSelectArgs, int) = {kv_select_long_kernel<0>, kv_select_long_kernel<1>, kv_select_long_kernel<2>,
                                                     kv_select_long_kernel<3>};
        for (auto k : digits) {
            launch(k, dim3((unsigned)((long)a.b * a.Hkv * chunks)), dim3(kSelThreads), 0, s, a, chunks);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    const dim3 grid(a.b * a.Hkv);
    if (a.P <= 64 * kWaveKeys) launch(kv_select_wave_kernel, grid, dim3(64), 0, s, a);
    else if (a.P <= 2048) launch(kv_select_kernel<256, 8, 8>, grid, dim3(256), 0, s, a);
    else if (a.P <= 8 * kSelThreads) launch(kv_select_kernel<kSelThreads, 8, 11>, grid, dim3(kSelThreads), 0, s, a);
    else if (a.P <= 16 * kSelThreads) launch(kv_select_kernel<kSelThreads, 16, 11>, grid, dim3(kSelThreads), 0, s, a);
    else launch(kv_select_kernel<kSelThreads, 0, 11>, grid, dim3(kSelThreads), 0, s, a);
    return hipGetLastError();
}

template <typename T, int DH, int THREADS, int SEG, int ROWS, int E, bool NEAR>
static hipError_t compact_as(const KvCompactArgs& a, hipStream_t s) {
    const int parts = DH * (int)sizeof(T) / SEG + DH / ROWS + (a.weights ? 1 : 0);
    launch(kv_compact_kernel<T, DH, THREADS, SEG, ROWS, E, NEAR>, dim3((unsigned)((long)parts * a.b * a.Hkv)), dim3(THREADS), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !NEAR) return e;
    const int per = kFarThreads / (DH * (int)sizeof(T) / 16) * kFarPasses, blocks = (std::min(a.n, a.P) + per - 1) / per;
    launch(kv_compact_far_kernel<T, DH>, dim3((unsigned)((long)blocks * a.b * a.Hkv)), dim3(kFarThreads), 0, s, a, blocks);
    return hipGetLastError();
}

template <typename T>
static hipError_t compact(const KvCompactArgs& a, hipStream_t s) {
    // Few heads: more threads and smaller parts, and from 16384 keys on K in two launches (4 heads x 128,
    // from memory: 131072 -> 32768 keys 155 us in 256 threads, 125 in 1024, 74 in two launches; 16384 ->
    // 8192: 42, 32 and 35; 8192 -> 3000, twice as many heads: 21, 21 and 24).
    const bool few = (long)a.b * a.Hkv * a.dh < 4096;
    const int n = std::min(a.n, a.P);
    if (few && n > 16384) return a.dh == 128 ? compact_as<T, 128, 1024, 32, 4, 2, true>(a, s) : compact_as<T, 64, 1024, 32, 4, 2, true>(a, s);
    if (few && n > 4096) return a.dh == 128 ? compact_as<T, 128, 1024, 32, 2, 2, false>(a, s) : compact_as<T, 64, 1024, 32, 2, 2, false>(a, s);
    return a.dh == 128 ? compact_as<T, 128, 256, 64, 8, 1, false>(a, s) : compact_as<T, 64, 256, 64, 8, 1, false>(a, s);
}

hipError_t launch_kv_compact(int dtype, const KvCompactArgs& a, hipStream_t s) {
    if (dtype == DARD_DTYPE_F32) return compact<float>(a, s);
    return dtype == DARD_DTYPE_BF16 ? compact<bf16_t>(a, s) : compact<uint8_t>(a, s);
}

}  // namespace dard
