// State-masked attention of a batch whose sequences share a prefix (Sec. 3.1,
// Sec. 3.2; the prefix caching of App. C.5 for a prompt that a whole batch has).
//
// out_r = sum_k e^(s_rk - L_r) v_k,  L_r = log sum_k e^(s_rk),  s_rk = scale q_r . k_k
// over the Ps shared keys, the keys of the row's own sequence, and of its block
// the keys that the state mask lets it see.  The softmax is taken in one pass
// with a running maximum and sum.
//
// The rows of all sequences and of all query heads of a KV head are one row
// space, sequence by sequence, so a tile of shared keys that a workgroup stages
// in LDS serves rows of as many sequences as fit: one position a sequence (two
// rows) fills matrix tiles that a launch per sequence would leave empty, and the
// shared keys are read once for 128 rows instead of once for two.  A workgroup
// takes 128 consecutive rows and walks the shared tiles, then the own tiles
// of each sequence among its rows; waves without rows of that sequence leave the
// tile out.  An own tile is 64 consecutive keys of a sequence's prefix and
// block, and one 64-bit word per row says which of them the row sees.
//
// A wave has 32 rows: S^T = K Q^T puts a row in a lane pair, so the softmax needs one
// exchange a tile, and P^T is the next product's operand where it stands.  Two waves a
// SIMD take turns at the matrix and the vector unit; every wave reads the whole K and V
// tile from LDS, which is what 32 rows a wave cost.  (64 rows a wave: 645 us against 566 for
// the long case below in the same bench, the compiler moves half of the accumulators
// between register files in every tile; half-step phases of wave groups, priorities and
// an interleaved half tile were worth nothing.)  Measured: 14336 rows x 4 heads of 128, 16384
// shared and up to 256 own keys 0.49 ms, 995 TFLOP/s: the matrix unit is busy in 48 % of a
// SIMD's cycles, vector instructions issue in 40 %.  128 rows x 32 heads, 32768 shared keys
// 158 us, 537 MB of K and V at 3.4 TB/s: 16 splits, two workgroups a CU, that wait for
// their tiles.  The same from an FP8 cache takes longer, 207 us for half the bytes: codes go
// through registers, V chunks by the path for a cache's end in every tile, and are widened
// between the products and the barrier.  Heads of 64: 4096 rows x 4 heads, 8192 shared and up
// to 256 own keys 68 us (FP8 87), 26 at the matrix unit's full rate.
#include <algorithm>
#include <type_traits>

#include "attention_tiles.h"
#include "common.h"
#include "launch.h"

namespace dard {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// The running maximum (log2 units) before a row has seen a score.  Any score
// that float32 holds lies above it or makes exp2 of the difference infinite, so
// a first tile always moves it; a hidden key's minus infinity still gives 0.
constexpr float kLeast = -3.402823466e38f;
constexpr float kBig = 256.f;        // a lane's probability sum over a tile that moves the running maximum
constexpr int kMaxSplit = 32;        // key splits across workgroups
constexpr int kFewPositions = kSharedFewPositions;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A tile of the walk: seq < 0 for shared keys, else the sequence (counted from
// the workgroup's first); keys k0 .. k0 + n - 1 of that cache; p the sequence's
// prefix length.  Uniform over the workgroup.
struct Tile {
    int seq, k0, n, p;
};

// The block keys among keys k0 .. k0 + 63 of a sequence with prefix p that a row
// with take-x words x sees, and every prefix key among them.
__device__ __forceinline__ uint64_t own_word(const uint64_t (&x)[kBlockWords], int B, int p, int k0) {
    const int s = k0 - p;                                    // block position of the tile's first key
    const uint64_t pre = s >= 0 ? 0ull : (s <= -64 ? ~0ull : (1ull << -s) - 1);
    return pre | bits64(x, B, s) | (~bits64(x, B, s - B) & range_mask(s - B, B));
}

// LDS: three K stages [64 keys][DH] and two V^T stages [DH][64 keys].  With two GROUPS of
// waves each has stages, and a half of the workgroup's tiles, of its own, and the first
// takes the second's results from LDS at the end: two waves a SIMD without a merge in memory.
constexpr int kWaves = 4, kRows = 32 * kWaves;   // of a workgroup

template <int DH, bool KV8, int GROUPS>
__global__ __launch_bounds__(64 * kWaves * GROUPS) __attribute__((amdgpu_waves_per_eu(2)))
void shared_attn_kernel(SharedAttnArgs a, int rowtiles, int nsplit) {
    constexpr int ROWS = kRows, TILE = kKeys * DH * 2;
    constexpr int NI = kKeys * DH / 8 / (64 * kWaves);       // 16-byte chunks of a tile that a thread copies
    static_assert(ROWS <= 128, "at most 64 sequences among the rows");
    using KVT = typename std::conditional<KV8, uint8_t, bf16_t>::type;
    typedef __attribute__((address_space(3))) void* lds_ptr;
    typedef __attribute__((address_space(1))) void* glb_ptr;
    __shared__ __attribute__((aligned(16))) char smem[GROUPS * 5 * TILE];   // (and the rows' results on their way out)

    const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave = wid % kWaves, group = wid / kWaves;     // (of its group)
    char* stages = smem + group * 5 * TILE;
    const int lr = lane & 31, eta = lane >> 5;
    // row tile fastest, then key split, then KV head, dealt to the XCDs in
    // contiguous runs: workgroups that read the same keys share an L2
    int bid = blockIdx.x;
    {
        const int total = gridDim.x, per = total >> 3, more = total & 7, x = bid & 7;
        bid = x * per + min(x, more) + (bid >> 3);
    }
    const int rt = bid % rowtiles, split = bid / rowtiles % nsplit, kvh = bid / rowtiles / nsplit;
    const int GQ = a.Hq / a.Hkv, R = 2 * a.B, RS = GQ * R;   // rows of a sequence: (position row, head), head fastest
    const int total_rows = a.b * RS;

    // ---- the walk: shared tiles, then the own tiles of sequences s0 ..; lane i
    // holds the prefix length of sequence s0 + i and the own tiles up to it
    const int s0 = rt * ROWS / RS;
    const int nseq = (min(rt * ROWS + ROWS, total_rows) - 1) / RS - s0 + 1;   // at most 64: RS >= 2
    const int nsh = (a.Ps + kKeys - 1) / kKeys;
    int plen = 0, upto = 0;
    if (lane < nseq) {
        plen = a.prefix ? min(max(a.prefix[s0 + lane], 0), a.P) : a.P;
        upto = (plen + R + kKeys - 1) / kKeys;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int below = __shfl_up(upto, o, 64);
        if (lane >= o) upto += below;
    }
    const int ntiles = nsh + __builtin_amdgcn_readlane(upto, 63);
    auto first_of = [&](int part) __attribute__((always_inline)) { return (int)((long long)ntiles * part / (nsplit * GROUPS)); };
    const int t_begin = first_of(split * GROUPS + group), t_end = first_of(split * GROUPS + group + 1);
    int steps = t_end - t_begin;                             // (of the group that has more)
    if constexpr (GROUPS == 2) steps = max(steps, first_of(split * 2 + 2 - group) - first_of(split * 2 + 1 - group));
    auto tile_at = [&](int t) __attribute__((always_inline)) {
        Tile d;
        if (t < nsh) {
            d.seq = -1;
            d.k0 = t * kKeys;
            d.n = min(kKeys, a.Ps - d.k0);
            d.p = 0;
        } else {
            const int u = t - nsh;
            const int i = __builtin_popcountll(__ballot(upto <= u));   // (lanes past the last sequence hold the total)
            d.seq = i;
            d.p = __builtin_amdgcn_readlane(plen, i);
            d.k0 = (u - (i ? __builtin_amdgcn_readlane(upto, i - 1) : 0)) * kKeys;
            d.n = min(kKeys, d.p + R - d.k0);
        }
        return d;
    };

    const KVT* ksh = reinterpret_cast<const KVT*>(a.ksh) + (size_t)kvh * a.cap_sh * DH;
    const KVT* vsh = reinterpret_cast<const KVT*>(a.vsh) + (size_t)kvh * a.cap_sh * DH;
    auto keys_of = [&](const Tile& d) __attribute__((always_inline)) {
        const KVT* base = d.seq < 0 ? ksh : reinterpret_cast<const KVT*>(a.k) + ((size_t)(s0 + d.seq) * a.Hkv + kvh) * a.cap * DH;
        return reinterpret_cast<const char*>(base + (size_t)d.k0 * DH);
    };
    auto values_of = [&](const Tile& d) __attribute__((always_inline)) {
        const KVT* base = d.seq < 0 ? vsh : reinterpret_cast<const KVT*>(a.v) + ((size_t)(s0 + d.seq) * a.Hkv + kvh) * a.cap * DH;
        return reinterpret_cast<const char*>(base + d.k0);
    };

    // ---- copies into LDS.  Chunk q = (wave NI + j) 64 + lane of the swizzled
    // image goes straight there (16 bytes a lane; an FP8 cache goes through
    // registers and is widened).  K rows past a tile's n keys are
    // left out (their scores are masked, whatever the stage held).  Values past them
    // come along where the cache holds 64 (their probabilities are 0, and infinities
    // and NaN are looked for in such tiles); past the cache's end nothing is read.
    // Addresses are a uniform part and 32 bits of a lane's own.
    uint32_t koff[NI];                                       // byte of the lane's chunk j in a K tile
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const int q = (wave * NI + j) * 64 + lane, r = q / (DH / 8);
        koff[j] = (uint32_t)(r * DH + 8 * ((q % (DH / 8)) ^ kswz<DH>(r))) * sizeof(KVT);
    }
    auto krow = [&](int j) __attribute__((always_inline)) { return ((wave * NI + j) * 64 + lane) / (DH / 8); };
    // V chunk j: row d = 8 (wave NI + j) + lane / 8, keys 8 c .. of the tile
    auto vchunk = [&](int j) __attribute__((always_inline)) { return ((lane & 7) ^ (lane >> 3) ^ (wave * NI + j)) & 7; };
    auto vrow = [&](const char* vt, int j, int vcap) __attribute__((always_inline)) {
        return vt + (size_t)(8 * (wave * NI + j)) * vcap * sizeof(KVT);
    };
    u32x2 kreg[NI], vreg[NI];
    auto load_k8 = [&](const Tile& t) __attribute__((always_inline)) {
        const char* kt = keys_of(t);
#pragma unroll
        for (int j = 0; j < NI; ++j)
            if (krow(j) < t.n) kreg[j] = *reinterpret_cast<const u32x2*>(kt + koff[j]);
    };
    auto commit_k8 = [&](const Tile& t, char* dst) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            if (krow(j) < t.n) *reinterpret_cast<uint4*>(dst + 16 * ((wave * NI + j) * 64 + lane)) = e4m3x8_to_bf16x8_scaled(kreg[j][0], kreg[j][1]);
        }
    };
    // (a V row starts at any byte: cap and the tile's first key may be odd)
    typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(1)));
    typedef uint64_t u64x2u __attribute__((ext_vector_type(2), aligned(2)));
    auto load_v8 = [&](const Tile& t) __attribute__((always_inline)) {
        const char* vt = values_of(t);
        const int vcap = t.seq < 0 ? a.cap_sh : a.cap;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int c = vchunk(j), have = vcap - t.k0 - 8 * c, back = have < 8 ? 8 - have : 0;   // keys of the row from here on
            uint64_t w = 0;
            if (back < 8 && vcap >= 8) {
                const u32x2u x = *reinterpret_cast<const u32x2u*>(vrow(vt, j, vcap) + ((uint32_t)(lane >> 3) * vcap + 8 * c) - back);
                w = (((uint64_t)x[1] << 32) | x[0]) >> (8 * back);
            }
            vreg[j] = u32x2{(uint32_t)w, (uint32_t)(w >> 32)};
        }
    };
    auto commit_v8 = [&](char* dst) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NI; ++j)
            *reinterpret_cast<uint4*>(dst + 16 * ((wave * NI + j) * 64 + lane)) = e4m3x8_to_bf16x8_scaled(vreg[j][0], vreg[j][1]);
    };
    auto issue_k = [&](const Tile& t, char* dst) __attribute__((always_inline)) {
        if constexpr (KV8) {
            load_k8(t);
            commit_k8(t, dst);
        } else {
            const char* kt = keys_of(t);
            auto copy = [&](int j) __attribute__((always_inline)) {
                __builtin_amdgcn_global_load_lds((glb_ptr)(kt + koff[j]), (lds_ptr)(dst + (wave * NI + j) * 1024), 16, 0, 0);
            };
            if (t.n == kKeys) {
#pragma unroll
                for (int j = 0; j < NI; ++j) copy(j);
                return;
            }
#pragma unroll
            for (int j = 0; j < NI; ++j)
                if (krow(j) < t.n) copy(j);
        }
    };
    auto issue_v = [&](const Tile& t, char* dst) __attribute__((always_inline)) {
        if constexpr (KV8) {
            load_v8(t);
            commit_v8(dst);
        } else {
            const char* vt = values_of(t);
            const int vcap = t.seq < 0 ? a.cap_sh : a.cap;
            const uint32_t row = (uint32_t)(lane >> 3) * vcap * 2;
            auto copy = [&](int j) __attribute__((always_inline)) {
                __builtin_amdgcn_global_load_lds((glb_ptr)(vrow(vt, j, vcap) + (row + 16 * vchunk(j))),
                                                 (lds_ptr)(dst + (wave * NI + j) * 1024), 16, 0, 0);
            };
            if (t.k0 + kKeys <= vcap) {
#pragma unroll
                for (int j = 0; j < NI; ++j) copy(j);
                return;
            }
#pragma unroll
            for (int j = 0; j < NI; ++j)
                if (t.k0 + 8 * vchunk(j) + 8 <= vcap) copy(j);
            // chunks that pass the cache's end: the last 8 keys of the row, shifted, or zeros
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int c = vchunk(j), back = 8 - (vcap - t.k0 - 8 * c);
                if (back <= 0) continue;
                uint64_t lo = 0, hi = 0;
                if (back < 8 && vcap >= 8) {
                    const u64x2u x = *reinterpret_cast<const u64x2u*>(vrow(vt, j, vcap) + (row + 16 * c) - 2 * back);
                    const int sh = 16 * (back & 3);
                    lo = back >= 4 ? x[1] >> sh : (sh ? (x[0] >> sh) | (x[1] << (64 - sh)) : x[0]);
                    hi = back >= 4 ? 0 : x[1] >> sh;
                }
                *reinterpret_cast<uint4*>(dst + 16 * ((wave * NI + j) * 64 + lane)) =
                    make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
            }
        }
    };
    // a cache of less than 8 keys has no 8 to read: element by element into the stage (the lane's own
    // chunks, after what issue_v or commit_v8 wrote there)
    auto tiny_v = [&](const Tile& t, char* dst) __attribute__((always_inline)) {
        const int vcap = t.seq < 0 ? a.cap_sh : a.cap;
        if (vcap >= 8) return;
        const char* vt = values_of(t);
#pragma unroll 1
        for (int j = 0; j < NI; ++j) {
#pragma unroll 1
            for (int e = 0; e < t.n && vchunk(j) == 0; ++e) {
                const KVT x = reinterpret_cast<const KVT*>(vrow(vt, j, vcap))[(lane >> 3) * vcap + e];
                uint16_t w;
                if constexpr (KV8) w = (uint16_t)e4m3x2_to_bf16x2<false>(x);
                else w = x;
                *reinterpret_cast<uint16_t*>(dst + 16 * ((wave * NI + j) * 64 + lane) + 2 * e) = w;
            }
        }
    };
    auto kst = [&](int i) __attribute__((always_inline)) { return stages + (i % 3) * TILE; };
    auto vst = [&](int i) __attribute__((always_inline)) { return stages + (3 + (i & 1)) * TILE; };
    // tiles of this step, the next and the one after it (none: n = 0)
    const Tile none = {-1, 0, 0, 0};
    Tile t0 = t_begin < t_end ? tile_at(t_begin) : none, t1 = t_begin + 1 < t_end ? tile_at(t_begin + 1) : none;
    if (t0.n) {
        issue_k(t0, kst(0));
        issue_v(t0, vst(0));
        tiny_v(t0, vst(0));
    }
    if (t1.n) issue_k(t1, kst(1));

    // ---- this lane's query row, its Q operand and its take-x words
    const int rho = rt * ROWS + 32 * wave + lr;
    const bool row_ok = rho < total_rows;
    const int rc = min(rho, total_rows - 1);
    const int seq = rc / RS, r = rc % RS / GQ, h = kvh * GQ + rc % GQ;
    const size_t orow = ((size_t)seq * R + r) * a.Hq + h;    // (sequence, row, head)
    // sequences of the wave's rows, counted from s0 (a wave past the last row has none)
    const int w_lo = __builtin_amdgcn_readfirstlane(seq) - s0, w_hi = __builtin_amdgcn_readlane(seq, 31) - s0;
    const bool w_any = rt * ROWS + 32 * wave < total_rows;
    bf16x8 qf[DH / 16];
#pragma unroll
    for (int c = 0; c < DH / 16; ++c)
        qf[c] = ld_bf16x8(reinterpret_cast<const bf16_t*>(a.q) + orow * DH + 16 * c + 8 * eta);
    // take-x words: the first kept, others read where a tile has block keys (they would
    // hold 6 registers through the loop).  Few positions: worked out here, behind the
    // first copies (a kernel of their own takes 3 to 4 us); the wave's sequences have at
    // most 16 / GQ + 2 B <= 48 of them, one a lane
    const int W = (a.B + 63) / 64;
    const uint64_t* sel = a.sel + ((size_t)seq * R + r) * W;
    uint64_t sel0 = 0;
    if (a.B > kFewPositions) {
        sel0 = sel[0];
    } else if (t_end > nsh) {
        const int at = min((s0 + w_lo) * a.B + lane, a.b * a.B - 1);
        const int st = a.state[at];
        const float cf = a.conf[at];
        const int base = (seq - s0 - w_lo) * a.B, i = r % a.B, si = __shfl(st, base + i, 64);
        const float ci = __shfl(cf, base + i, 64);
        for (int j = 0; j < a.B; ++j)
            if (take_x(si, __shfl(st, base + j, 64), ci, __shfl(cf, base + j, 64), i, j, r >= a.B, a.flags)) sel0 |= 1ull << j;
    }
    const float sl2 = a.scale * kLog2e;
    // K row pi(lr) of each 32-key block, V^T row lr: operand addresses inside a
    // stage; a chunk or a block of rows further is an XOR or an offset
    const uint32_t kaddr0 = 16 * kslot<DH>(swap23(lr), eta), vaddr0 = 16 * vslot(lr, eta);

    floatx16 o[DH / 32];
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[d][v] = 0.f;
    float m_run = kLeast, l_run = 0.f;

    // S^T = K Q^T: value v of block kb is key 32 kb + 16 (v / 8) + 8 eta + v % 8
    auto scores = [&](const char* ks, floatx16 (&sc)[2]) __attribute__((always_inline)) {
        // (two chains of products in turn; operand reads run eight ahead)
        constexpr int NF = DH / 8;
        const uint32_t kb0 = (uint32_t)(ks - smem) + kaddr0;
        bf16x8 kf[NF];
#pragma unroll
        for (int i = 0; i < NF; ++i)
            kf[i] = *reinterpret_cast<const bf16x8*>(smem + ((kb0 ^ (32u * (i >> 1))) + (i & 1) * 32 * DH * 2));
#pragma unroll
        for (int v = 0; v < 16; ++v) sc[0][v] = sc[1][v] = 0.f;
#pragma unroll
        for (int i = 0; i < NF; ++i) sc[i & 1] = mfma32x32x16(kf[i], qf[i >> 1], sc[i & 1]);
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
        if constexpr (NF == 16) {
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    };
    auto vfrag = [&](const char* vs, int d, int st) __attribute__((always_inline)) {
        const uint32_t vb0 = (uint32_t)(vs - smem) + vaddr0;
        return *reinterpret_cast<const bf16x8*>(smem + ((vb0 ^ (32u * (st ^ (2 * (d & 1))))) + d * 32 * kKeys * 2));
    };
    // mask, online softmax and O^T += V^T P^T.  Probabilities are taken against the
    // running maximum as it stands, and once more against the tile's where a lane's
    // sum of them passes kBig (or is NaN).  They are rounded to bf16 for the matrix
    // unit (2^-8 of each at most); their sum is not.
    auto softmax_pv = [&](floatx16 (&sc)[2], const Tile& t, const char* vs) __attribute__((always_inline)) {
        // whole: every row of the wave sees every key of the tile
        const bool whole = t.n == kKeys && (t.seq < 0 || (w_lo == w_hi && t.k0 + kKeys <= t.p));
        uint64_t vis = ~0ull;
        if (!whole) {
            if (t.seq < 0) vis = (1ull << t.n) - 1;          // (n < 64 here)
            else {
                uint64_t xw[kBlockWords];
#pragma unroll
                for (int q = 0; q < kBlockWords; ++q) xw[q] = q == 0 ? sel0 : (q < W ? sel[q] : 0ull);
                vis = seq - s0 == t.seq ? own_word(xw, a.B, t.p, t.k0) : 0ull;
            }
            const uint64_t ww = vis >> (8 * eta);
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (!((ww >> (32 * kb + 16 * (v >> 3) + (v & 7))) & 1ull)) sc[kb][v] = -INFINITY;
        }
        float psum = 0.f;
        bf16x8 pb[2][2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const float p = __builtin_amdgcn_exp2f(fmaf(sc[kb][v], sl2, -m_run));
                psum += p;
                pb[kb][v >> 3][v & 7] = (__bf16)p;
            }
        if (__ballot(!(psum <= kBig))) {
            float mt = sc[0][0];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int v = 0; v < 16; ++v) mt = fmaxf(mt, sc[kb][v]);
            mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
            const float m_new = fmaxf(m_run, mt * sl2);      // sl2 > 0: the maximum commutes with the scale
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
#pragma unroll
            for (int d = 0; d < DH / 32; ++d) o[d] *= alpha;
            l_run *= alpha;
            m_run = m_new;
            psum = 0.f;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(sc[kb][v], sl2, -m_run));
                    psum += p;
                    pb[kb][v >> 3][v & 7] = (__bf16)p;
                }
        }
        l_run += psum;
        // An infinity or NaN among the values of a tile that not every row sees whole
        // must not reach the rows that do not see its key (0 times it is NaN), nor may
        // one behind the tile's keys: such elements are left out of the product and
        // added row by row.
        bool odd = false;
        if (!whole) {
            uint32_t top = 0;
#pragma unroll
            for (int d = 0; d < DH / 32; ++d)
#pragma unroll
                for (int st = 0; st < 4; ++st) {
                    const u32x4 w = __builtin_bit_cast(u32x4, vfrag(vs, d, st));
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        top |= ((w[e] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;   // exponent all ones
                }
            odd = __ballot(top != 0) != 0;
        }
#pragma unroll
        for (int d = 0; d < DH / 32; ++d) {
            bf16x8 vf[4];
#pragma unroll
            for (int st = 0; st < 4; ++st) vf[st] = vfrag(vs, d, st);
            if (odd) {
#pragma unroll
                for (int st = 0; st < 4; ++st) {
                    u32x4 w = __builtin_bit_cast(u32x4, vf[st]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t m = ((w[e] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;   // bit 15 of an odd half
                        w[e] &= ~(m | (m - (m >> 15)));
                    }
                    vf[st] = __builtin_bit_cast(bf16x8, w);
                }
            }
#pragma unroll
            for (int st = 0; st < 4; ++st) o[d] = mfma32x32x16(vf[st], pb[st >> 1][st & 1], o[d]);
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
        }
        if (odd) {
            for (int key = 0; key < t.n; ++key) {
                const bool sees = (vis >> key) & 1ull;
                if (!__ballot(sees)) continue;
                // the row's probability of this key, from the lane of the row that holds it
                const int kb = key >> 5, e = (key & 7) + 8 * ((key >> 4) & 1), from = lr + 32 * ((key >> 3) & 1);
                float pk = 0.f;
#pragma unroll
                for (int b2 = 0; b2 < 2; ++b2)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (b2 == kb && v == e) pk = (float)pb[b2][v >> 3][v & 7];
                pk = __shfl(pk, from, 64);
#pragma unroll
                for (int d = 0; d < DH / 32; ++d)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int dim = 32 * d + 8 * (v >> 2) + 4 * eta + (v & 3);
                        const bf16_t w = *reinterpret_cast<const bf16_t*>(vs + 16 * vslot(dim, key >> 3) + 2 * (key & 7));
                        o[d][v] += sees && (w & 0x7F80u) == 0x7F80u ? pk * bf2f(w) : 0.f;
                        __builtin_amdgcn_sched_barrier(0);   // (a rare path: as few registers as it can)
                    }
            }
        }
    };
    // rows of this wave that the tile can concern
    auto concerns = [&](const Tile& t) __attribute__((always_inline)) {
        return w_any && (GROUPS == 1 || t.n) && (t.seq < 0 || (t.seq >= w_lo && t.seq <= w_hi));
    };

    // ---- main loop: V one step ahead of its use, K two.  A step ends by waiting for
    // every copy but the newest K tile's and publishing them with the barrier, which
    // also retires every wave's reads of the stages that the next step overwrites.
    // Copies complete in order, so V goes first; a ragged K tile issues fewer copies
    // than the count assumes, so then all are waited for.
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    for (int it = 0; it < steps; ++it) {
        const Tile t2 = t_begin + it + 2 < t_end ? tile_at(t_begin + it + 2) : none;
        if constexpr (KV8) {
            if (t1.n) load_v8(t1);
            if (t2.n) load_k8(t2);
        } else {
            if (t1.n) {
                issue_v(t1, vst(it + 1));
                tiny_v(t1, vst(it + 1));
            }
            if (t2.n) issue_k(t2, kst(it + 2));
        }
        if (concerns(t0)) {
            floatx16 sc[2];
            scores(kst(it), sc);
            softmax_pv(sc, t0, vst(it));
        }
        if constexpr (KV8) {
            if (t1.n) {
                commit_v8(vst(it + 1));
                tiny_v(t1, vst(it + 1));
            }
            if (t2.n) commit_k8(t2, kst(it + 2));
            __builtin_amdgcn_s_waitcnt(0);
        } else {
            if (t2.n == kKeys) __builtin_amdgcn_s_waitcnt(waitcnt_vm(NI));
            else __builtin_amdgcn_s_waitcnt(0);
        }
        wg_barrier();
        t0 = t1;
        t1 = t2;
    }

    // ---- the second group's results, through its stages, into the first's (lane by lane:
    // both hold the same rows)
    if constexpr (GROUPS == 2) {
        constexpr int NO = DH / 8;                           // 16-byte pieces of a lane
        char* at = smem + 5 * TILE + wave * NO * 1024 + lane * 16;
        float2* ml = reinterpret_cast<float2*>(smem + 5 * TILE + kWaves * NO * 1024) + wave * 64 + lane;
        if (group == 1) {
#pragma unroll
            for (int i = 0; i < NO; ++i)
                *reinterpret_cast<floatx4*>(at + i * 1024) =
                    floatx4{o[i >> 2][4 * (i & 3)], o[i >> 2][4 * (i & 3) + 1], o[i >> 2][4 * (i & 3) + 2], o[i >> 2][4 * (i & 3) + 3]};
            *ml = make_float2(m_run, l_run);
        }
        __syncthreads();
        if (group == 1) return;
        const float2 v = *ml;
        const float m_new = fmaxf(m_run, v.x), f0 = __builtin_amdgcn_exp2f(m_run - m_new), f1 = __builtin_amdgcn_exp2f(v.x - m_new);
        m_run = m_new;
        l_run = l_run * f0 + v.y * f1;
#pragma unroll
        for (int i = 0; i < NO; ++i) {
            const floatx4 x = *reinterpret_cast<const floatx4*>(at + i * 1024);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i >> 2][4 * (i & 3) + e] = o[i >> 2][4 * (i & 3) + e] * f0 + x[e] * f1;
        }
    }

    // ---- epilogue: the two lanes of a row hold disjoint keys; a lane holds dims
    // 32 d + 8 j + 4 eta + {0..3}.  Rows go out through the wave's part of the LDS, so
    // that a store covers whole rows (16-byte pieces of 32 rows at a time took 7 us
    // of a call with 512 workgroups); chunk c of row r sits in slot c ^ r.
    const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
    const bool whole = nsplit == 1;
    const float inv = !whole ? 1.f : (l_tot == 0.f ? 0.f : 1.f / l_tot);   // (every score minus infinity: zeros)
    constexpr int FCH = DH / 4;                              // 16-byte chunks of a row in fp32
    char* own = stages + wave * 32 * DH * 4;
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = 8 * d + 2 * j + eta;
            *reinterpret_cast<floatx4*>(own + 16 * (lr * FCH + (c ^ (lr & (FCH - 1))))) =
                floatx4{o[d][4 * j] * inv, o[d][4 * j + 1] * inv, o[d][4 * j + 2] * inv, o[d][4 * j + 3] * inv};
        }
    const size_t nrow = (size_t)total_rows * a.Hkv;          // (b R Hq)
    if (eta == 0 && row_ok) {
        if (!whole)
            *reinterpret_cast<float2*>(a.part + (size_t)nsplit * nrow * DH + ((size_t)split * nrow + orow) * 2) = make_float2(m_run, l_tot);
        else if (a.lse)
            a.lse[orow] = l_tot == 0.f ? -INFINITY : (m_run + __log2f(l_tot)) * kLn2;
    }
    // a lane takes 8 values of a row, the row's place from the row's own lane
    constexpr int EPL = DH / 8, RPP = 64 / EPL;              // lanes a row (8 values each), rows a pass
    const int c8 = lane % EPL;
#pragma unroll
    for (int i = 0; i < 32 / RPP; ++i) {
        const int row = i * RPP + lane / EPL;
        const floatx4 x = *reinterpret_cast<const floatx4*>(own + 16 * (row * FCH + ((2 * c8) ^ (row & (FCH - 1)))));
        const floatx4 y = *reinterpret_cast<const floatx4*>(own + 16 * (row * FCH + ((2 * c8 + 1) ^ (row & (FCH - 1)))));
        const uint32_t to = __shfl((uint32_t)orow, row, 64);  // (rows times heads are under 2^31)
        if (rt * ROWS + 32 * wave + row >= total_rows) continue;
        if (whole) {
            bf16x8 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) { w[e] = (__bf16)x[e]; w[4 + e] = (__bf16)y[e]; }
            *reinterpret_cast<bf16x8*>(reinterpret_cast<bf16_t*>(a.out) + (size_t)to * DH + 8 * c8) = w;
        } else {
            float* po = a.part + ((size_t)split * nrow + to) * DH + 8 * c8;
            *reinterpret_cast<floatx4*>(po) = x;
            *reinterpret_cast<floatx4*>(po + 4) = y;
        }
    }
}

// Merge of key splits: out = sum_s o_s 2^(m_s - M) / sum_s l_s 2^(m_s - M) in
// split order, eight at a time (their loads go out together).  A thread per (row,
// head, 4 dims).
template <int DH, typename T>
__global__ __launch_bounds__(256) void shared_attn_combine_kernel(const float* __restrict__ part, int ns, size_t nrow,
                                                                  T* __restrict__ out, float* __restrict__ lse) {
    const size_t t = (size_t)blockIdx.x * 256 + threadIdx.x, row = t / (DH / 4);
    const int q4 = t % (DH / 4);
    if (row >= nrow) return;
    const float2* ml = reinterpret_cast<const float2*>(part + (size_t)ns * nrow * DH);
    float M = kLeast, l = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < ns; s += 8) {
        float2 v[8];
        floatx4 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at = min(s + i, ns - 1);
            v[i] = ml[at * nrow + row];
            x[i] = reinterpret_cast<const floatx4*>(part + (at * nrow + row) * DH)[q4];
        }
        float top = M;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, v[i].x);
        const float f0 = __builtin_amdgcn_exp2f(M - top);
        l *= f0;
        acc *= f0;
        M = top;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (s + i < ns) {
                const float f = __builtin_amdgcn_exp2f(v[i].x - M);
                l += v[i].y * f;
                acc += x[i] * f;
            }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if constexpr (sizeof(T) == 2) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        bf16x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (__bf16)(acc[e] * inv);
        *reinterpret_cast<bf16x4*>(out + row * DH + 4 * q4) = w;
    } else {
        st_f4(out + row * DH + 4 * q4, acc * inv);
    }
    if (lse && q4 == 0) lse[row] = l == 0.f ? -INFINITY : (M + __log2f(l)) * kLn2;
}

// fp32, on v_mfma_f32_16x16x4_f32: a workgroup takes 16 rows of the same row
// space; its four waves take interleaved tiles of 32 keys, shared ones first, and
// merge through LDS in wave order.  S^T = K Q^T leaves lane l (token l % 16, g = l / 16)
// with keys 4g .. 4g + 3, and the B operand of step e of O^T += V^T P^T is key
// 4g + e, so probabilities are used where they are.  K and V are loaded where they are used,
// by a single wave a SIMD: 256 rows x 32 heads of 128, 2048 shared and up to 128 own keys 170 us
// (59 at the matrix unit's full rate); 2048 rows x 4 heads of 64, 4096 and up to 128 134 (58).
constexpr int kWavesF = 4, kKeysF = 32;

template <int DH>
__global__ __launch_bounds__(64 * kWavesF) void shared_attn_f32_kernel(SharedAttnArgs a, int rowtiles, int nsplit) {
    constexpr int NC = DH / 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane & 15, g = lane >> 4;
    int bid = blockIdx.x;
    {
        const int total = gridDim.x, per = total >> 3, more = total & 7, x = bid & 7;
        bid = x * per + min(x, more) + (bid >> 3);
    }
    const int rt = bid % rowtiles, split = bid / rowtiles % nsplit, kvh = bid / rowtiles / nsplit;
    const int GQ = a.Hq / a.Hkv, R = 2 * a.B, RS = GQ * R, total_rows = a.b * RS;
    const int s0 = rt * 16 / RS, nseq = (min(rt * 16 + 16, total_rows) - 1) / RS - s0 + 1;   // at most 8
    const int nsh = (a.Ps + kKeysF - 1) / kKeysF;
    int plen = 0, upto = 0;
    if (lane < nseq) {
        plen = a.prefix ? min(max(a.prefix[s0 + lane], 0), a.P) : a.P;
        upto = (plen + R + kKeysF - 1) / kKeysF;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int below = __shfl_up(upto, o, 64);
        if (lane >= o) upto += below;
    }
    const int ntiles = nsh + __builtin_amdgcn_readlane(upto, 63);
    const int t_begin = (int)((long long)ntiles * split / nsplit), t_end = (int)((long long)ntiles * (split + 1) / nsplit);

    const int rho = rt * 16 + lr, rc = min(rho, total_rows - 1);
    const int seq = rc / RS, r = rc % RS / GQ, h = kvh * GQ + rc % GQ;
    const size_t orow = ((size_t)seq * R + r) * a.Hq + h;
    floatx4 qf[NC], o[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        qf[c] = ld_f4(reinterpret_cast<const float*>(a.q) + orow * DH + 16 * c + 4 * g);
        o[c] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const int i = r % a.B;
    const bool shadow = r >= a.B;
    const uint8_t* st = a.state + (size_t)seq * a.B;
    const float* cf = a.conf + (size_t)seq * a.B;
    const int si = st[i];
    const float ci = cf[i], sl2 = a.scale * kLog2e;
    float m = kLeast, l = 0.f;
    for (int t = t_begin + wave; t < t_end; t += kWavesF) {
        int k0, nk, tseq = -1, p = 0;
        if (t < nsh) {
            k0 = t * kKeysF;
            nk = a.Ps;
        } else {
            const int u = t - nsh, q = __builtin_popcountll(__ballot(upto <= u));
            tseq = s0 + q;
            p = __builtin_amdgcn_readlane(plen, q);
            k0 = (u - (q ? __builtin_amdgcn_readlane(upto, q - 1) : 0)) * kKeysF;
            nk = p + R;
        }
        const size_t head = tseq < 0 ? (size_t)kvh : (size_t)tseq * a.Hkv + kvh;
        const int vcap = tseq < 0 ? a.cap_sh : a.cap;
        const float* kk = reinterpret_cast<const float*>(tseq < 0 ? a.ksh : a.k) + head * vcap * DH;
        const float* vv = reinterpret_cast<const float*>(tseq < 0 ? a.vsh : a.v) + head * vcap * DH;
        floatx4 sc[2], vf[2][NC];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const float* kr = kk + (size_t)min(k0 + 16 * b + lr, nk - 1) * DH + 4 * g;
            floatx4 kf[NC];
#pragma unroll
            for (int c = 0; c < NC; ++c) kf[c] = ld_f4(kr + 16 * c);
            const int kv = k0 + 16 * b + 4 * g;              // (keys past the last one read as zero)
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const float* vr = vv + (size_t)(16 * c + lr) * vcap + kv;
                if (kv + 4 <= nk) {
                    vf[b][c] = ld_f4(vr);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) vf[b][c][e] = kv + e < nk ? vr[e] : 0.f;
                }
            }
            sc[b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[b] = mfma16x16x4f(kf[c][e], qf[c][e], sc[b]);
        }
        float mt = m;
        uint32_t vis = 0;                                    // bit 4b + e: the row sees key k0 + 16b + 4g + e
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int key = k0 + 16 * b + 4 * g + e;
                bool see = key < nk && (tseq < 0 || tseq == seq);
                if (see && tseq >= 0 && key >= p) {
                    const int j = key - p, jj = j < a.B ? j : j - a.B;
                    see = take_x(si, st[jj], ci, cf[jj], i, jj, shadow, a.flags) == (j < a.B);
                }
                sc[b][e] *= sl2;
                if (see) { vis |= 1u << (4 * b + e); mt = fmaxf(mt, sc[b][e]); }
            }
        mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
        mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
        const float alpha = __builtin_amdgcn_exp2f(m - mt);
        float ps = 0.f;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float pe = (vis >> (4 * b + e)) & 1u ? __builtin_amdgcn_exp2f(sc[b][e] - mt) : 0.f;
                sc[b][e] = pe;
                ps += pe;
            }
        l = l * alpha + ps;
        m = mt;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[c] *= alpha;
        // a key that a row does not see adds nothing to it, whatever V holds there
        bool odd = false;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) odd |= !(fabsf(vf[b][c][e]) < INFINITY);
        if (!__any(odd)) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[c] = mfma16x16x4f(vf[b][c][e], sc[b][e], o[c]);
        } else {
            for (int key = 0; key < kKeysF; ++key) {
                const int b = key >> 4, gk = (key >> 2) & 3, e = key & 3;
                float pe = 0.f;
#pragma unroll
                for (int b2 = 0; b2 < 2; ++b2)
#pragma unroll
                    for (int e2 = 0; e2 < 4; ++e2)
                        if (b2 == b && e2 == e) pe = sc[b2][e2];
                pe = __shfl(pe, lr + 16 * gk, 64);
                const uint32_t w = __shfl((int)vis, lr + 16 * gk, 64);
                if (!((w >> (4 * b + e)) & 1u)) continue;
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int d = 0; d < 4; ++d)
                        o[c][d] += pe * vv[(size_t)(16 * c + 4 * g + d) * vcap + k0 + key];
            }
        }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    __shared__ floatx4 po[kWavesF][NC][64];
    __shared__ float pm[kWavesF][16], pl[kWavesF][16];
#pragma unroll
    for (int c = 0; c < NC; ++c) po[wave][c][lane] = o[c];
    if (g == 0) { pm[wave][lr] = m; pl[wave][lr] = l; }
    __syncthreads();
    float M = pm[0][lr];
#pragma unroll
    for (int w = 1; w < kWavesF; ++w) M = fmaxf(M, pm[w][lr]);
    float f[kWavesF], lt = 0.f;
#pragma unroll
    for (int w = 0; w < kWavesF; ++w) {
        f[w] = __builtin_amdgcn_exp2f(pm[w][lr] - M);
        lt += pl[w][lr] * f[w];
    }
    if (rho >= total_rows) return;
    const size_t nrow = (size_t)total_rows * a.Hkv;
    const float inv = nsplit > 1 ? 1.f : (lt == 0.f ? 0.f : 1.f / lt);
    float* dst = nsplit > 1 ? a.part + ((size_t)split * nrow + orow) * DH : reinterpret_cast<float*>(a.out) + orow * DH;
    for (int c = wave; c < NC; c += kWavesF) {
        floatx4 v = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWavesF; ++w) v += po[w][c][lane] * f[w];
        st_f4(dst + 16 * c + 4 * g, v * inv);
    }
    if (wave == 0 && g == 0) {
        if (nsplit > 1)
            *reinterpret_cast<float2*>(a.part + (size_t)nsplit * nrow * DH + ((size_t)split * nrow + orow) * 2) = make_float2(M, lt);
        else if (a.lse)
            a.lse[orow] = lt == 0.f ? -INFINITY : (M + __log2f(lt)) * kLn2;
    }
}

struct SharedCfg {
    int rowtiles, ns;
    int groups;   // of waves in a workgroup (bf16, FP8)
};

// Key splits, and a second group of waves in every workgroup: what is least by estimate.
// A step of a tile (fp32: of a tile for each of four waves) takes so many us for one
// workgroup on a CU, for each of two, and for a pair of groups; a split 4 us for the merge
// and 1040 bytes a row written and read at 5 TB/s, a second group 1.  So a pair is taken
// where workgroups leave half of the chip empty and a merge would cost more than the steps
// of two workgroups, which drift apart, save over those of a pair.  The constants are of heads
// of 128 and stand for 64 too (unmeasured there).  Measured (bf16; whole /
// whole in pairs / in two splits): 1024 rows x 32 heads, 10 tiles 38 / 34 / 46 us, 30 tiles
// 62 / 53 / 62, 82 tiles 151 / 126 / 126, 254 tiles 445 / 388 / 363; FP8 57 / 42 / 55,
// 99 / 71 / 81, 272 / 175 / 176, 661 / 459 / 445.  16 rows x 32 heads, 13 tiles: 14 us in 13
// splits, 17 in 6; fp32, 128 rows x 4 heads, 19 tiles: 11 us in 5 splits, 14 in 3, 20 whole.
SharedCfg shared_cfg(int dtype, int b, int B, int Hq, int Hkv, int Ps, int P) {
    SharedCfg c{};
    const long rows = (long)b * 2 * B * (Hq / Hkv), RS = 2L * B * (Hq / Hkv);
    const bool f32 = dtype == DARD_DTYPE_F32;
    const long per = f32 ? 16 : kRows, keys = f32 ? kKeysF : kKeys;
    c.rowtiles = (int)((rows + per - 1) / per);
    const long wgs = (long)c.rowtiles * Hkv;
    // sequences among a workgroup's rows, at most (they may begin inside it)
    const long seqs = std::min<long>(b, per % RS == 0 ? per / RS : RS % per == 0 ? 1 : (per - 2) / RS + 2);
    const long tiles = ((long)Ps + keys - 1) / keys + seqs * (((long)P + 2 * B + keys - 1) / keys);
    const bool kv8 = dtype == DARD_DTYPE_BF16_KV_FP8;
    const double alone = f32 ? 2.5 : kv8 ? 3.0 : 1.75, two = kv8 ? 3.3 : 2.7, pair = kv8 ? 3.55 : 3.0;
    const long step = f32 ? kWavesF : 1, fit = f32 ? 256 : 512;
    double best = 0;
    for (long ns = 1; ns <= kMaxSplit && (ns == 1 || (ns * wgs <= fit && (ns - 1) * step < tiles)); ++ns) {
        const long most = (tiles + ns - 1) / ns;             // of a split
        const double us = (double)((most + step - 1) / step) * (f32 || ns * wgs <= 256 ? alone : two) +
                          (ns > 1 ? 4 + (double)ns * rows * Hkv * 0.00021 : 0);
        if (ns == 1 || us < best) {
            best = us;
            c.ns = (int)ns;
        }
    }
    c.groups = 1;
    if (!f32 && wgs <= 256 && tiles > 1 && (double)((tiles + 1) / 2) * pair + 1 < best) {
        c.ns = 1;
        c.groups = 2;
    }
    return c;
}

}  // namespace

size_t shared_attention_partial_floats(int dtype, int b, int B, int Hq, int Hkv, int dh, int Ps, int P) {
    const SharedCfg c = shared_cfg(dtype, b, B, Hq, Hkv, Ps, P);
    return c.ns <= 1 ? 0 : (size_t)c.ns * b * 2 * B * Hq * (dh + 2);
}

template <int DH>
static hipError_t launch_shared(int dtype, const SharedAttnArgs& a, hipStream_t s) {
    const SharedCfg c = shared_cfg(dtype, a.b, a.B, a.Hq, a.Hkv, a.Ps, a.P);
    const dim3 grid((unsigned)((long)c.rowtiles * a.Hkv * c.ns));
    const bool f32 = dtype == DARD_DTYPE_F32;
    if (f32) {
        launch(shared_attn_f32_kernel<DH>, grid, dim3(64 * kWavesF), 0, s, a, c.rowtiles, c.ns);
    } else {
        const bool kv8 = dtype == DARD_DTYPE_BF16_KV_FP8;
        void (*k)(SharedAttnArgs, int, int) = c.groups == 2 ? (kv8 ? shared_attn_kernel<DH, true, 2> : shared_attn_kernel<DH, false, 2>)
                                                            : (kv8 ? shared_attn_kernel<DH, true, 1> : shared_attn_kernel<DH, false, 1>);
        launch(k, grid, dim3(64 * kWaves * c.groups), 0, s, a, c.rowtiles, c.ns);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || c.ns == 1) return e;
    const size_t nrow = (size_t)a.b * 2 * a.B * a.Hq;
    const dim3 cg((unsigned)((nrow * (DH / 4) + 255) / 256));
    if (f32)
        launch(shared_attn_combine_kernel<DH, float>, cg, dim3(256), 0, s, (const float*)a.part, c.ns, nrow, (float*)a.out, a.lse);
    else
        launch(shared_attn_combine_kernel<DH, bf16_t>, cg, dim3(256), 0, s, (const float*)a.part, c.ns, nrow, (bf16_t*)a.out, a.lse);
    return hipGetLastError();
}

hipError_t launch_shared_attention(int dtype, const SharedAttnArgs& a, hipStream_t s) {
    return a.dh == 128 ? launch_shared<128>(dtype, a, s) : launch_shared<64>(dtype, a, s);
}

}  // namespace dard
