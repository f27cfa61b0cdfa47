// State-masked attention over an MXFP4 key/value cache (Sec. 3.1, Sec. 3.2;
// the block-scaled form of the prefix cache of App. C.5).
//
// Flash-style on v_mfma_f32_32x32x16_bf16: S^T = K Q^T and O^T += V^T P^T over
// tiles of 32 keys, with a running maximum and sum per query row.  The rows of
// all query heads of a KV head are one row space.  A wave takes 32 JT rows and
// whole key tiles on its own: codes go from memory straight to its registers in
// operand order and are widened to bf16 there by the scaled conversions (exact:
// an E2M1 value times a power of two), so the main loop has no LDS traffic and
// no barrier.  The four waves of a workgroup take interleaved tiles and merge
// through LDS; long key ranges are also split over workgroups (fp32 partials,
// merged in split order by a second kernel).
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
#include "launch.h"
#include "mx.h"

namespace dard {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFloor = -1e30f;   // running-max floor (log2 units): exp2 of anything below it is 0
constexpr int kTileKeys = 32;
constexpr int kVisWords = 2 * kMaxBlock / 32 + 2;   // 32-bit words of a row's visibility, padded

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return (uint32_t)f2bf(lo) | ((uint32_t)f2bf(hi) << 16);
}

__device__ __forceinline__ bf16x8 as_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_bit_cast(bf16x8, make_uint4(a, b, c, d));
}

// Codes and scales of one key tile as a lane loads them.
template <int DH> struct Raw {
    uint4 k[DH / 64];     // this lane's half key
    uint32_t ks;          // its scales (one byte per 32 dims)
    uint4 v[2];           // 8 keys of this lane's dims, steps m = 0, 1
    uint2 vs[2];          // their scales
};

template <int DH>
__device__ __forceinline__ Raw<DH> load_tile(const MxAttnArgs& a, size_t row0, int k0, int lane) {
    const int lr = lane & 31, eta = lane >> 5;
    Raw<DH> t;
    const size_t key = row0 + k0 + ((lr & ~12) | ((lr & 4) << 1) | ((lr & 8) >> 1));
    const uint4* kp = reinterpret_cast<const uint4*>(a.kc + key * (DH / 2) + eta * (DH / 4));
#pragma unroll
    for (int i = 0; i < DH / 64; ++i) t.k[i] = kp[i];
    if constexpr (DH == 128) t.ks = reinterpret_cast<const uint16_t*>(a.ks)[key * 2 + eta];
    else t.ks = a.ks[key * 2 + eta];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const size_t grp = ((row0 + k0) >> 3) + 2 * m + eta;
        const int quad = DH == 128 ? lr : lr >> 1, blk = DH == 128 ? lr >> 3 : lr >> 4;
        t.v[m] = *reinterpret_cast<const uint4*>(a.vc + (grp * (DH / 4) + quad) * 16);
        t.vs[m] = *reinterpret_cast<const uint2*>(a.vs + (grp * (DH / 32) + blk) * 8);
    }
    return t;
}

// Does the row (position i, shadow) see key idx of the block (x keys, then s keys)?
__device__ __forceinline__ bool sees(const uint8_t* st, const float* cf, int i, bool shadow, int idx, int B,
                                     uint32_t flags) {
    if (idx >= 2 * B) return false;
    const int j = idx < B ? idx : idx - B;
    return take_x(st[i], st[j], cf[i], cf[j], i, j, shadow, flags) == (idx < B);
}

template <int DH, int JT>
__global__ __launch_bounds__(256) void attn_mx_kernel(MxAttnArgs a, int rowtiles, int tps) {
    constexpr int NJ = DH / 16, NT = DH / 32;
    __shared__ __attribute__((aligned(16))) float smem[4 * NT * 4 * 64 * 4];   // O of one row tile of the four waves
    __shared__ float ml[4][JT][2][32];
    __shared__ uint32_t vis[32 * JT][kVisWords];
    __shared__ uint8_t sst[kMaxBlock];
    __shared__ float scf[kMaxBlock];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane & 31, eta = lane >> 5;
    const int rt = blockIdx.x % rowtiles, kvh = blockIdx.x / rowtiles % a.Hkv, s = blockIdx.x / rowtiles / a.Hkv;
    const int R = 2 * a.B, GQ = a.Hq / a.Hkv, nrows = GQ * R;
    int P = a.P;
    if (a.prefix) P = min(max(__builtin_amdgcn_readfirstlane(a.prefix[s]), 0), a.P);
    const int nkeys = P + R, ntiles = (nkeys + kTileKeys - 1) / kTileKeys;
    const int t0 = blockIdx.y * tps, t1 = min(ntiles, t0 + tps);

    // visibility strings of the workgroup's rows, where its keys reach the block
    if (t1 * kTileKeys > P && t0 < t1) {
        for (int i = threadIdx.x; i < a.B; i += 256) {
            sst[i] = a.state[(size_t)s * a.B + i];
            scf[i] = a.conf[(size_t)s * a.B + i];
        }
        __syncthreads();
        const int words = (R + 31) / 32;
        for (int i = threadIdx.x; i < 32 * JT * kVisWords; i += 256) {
            const int row = i / kVisWords, w = i % kVisWords;
            uint32_t bits = 0;
            const int rho = rt * 32 * JT + row;
            if (w < words && rho < nrows) {
                const int r = rho % R;
                const bool shadow = r >= a.B;
                const int pos = shadow ? r - a.B : r;
                for (int b = 0; b < 32; ++b)
                    bits |= (uint32_t)sees(sst, scf, pos, shadow, 32 * w + b, a.B, a.flags) << b;
            }
            vis[row][w] = bits;
        }
    }
    __syncthreads();

    // this lane's query rows: dims of the half eta
    bf16x8 q[JT][NJ];
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) {
        const int rho = min(rt * 32 * JT + 32 * jt + lr, nrows - 1);
        const bf16_t* qp = a.q + (((size_t)s * R + rho % R) * a.Hq + kvh * GQ + rho / R) * DH + eta * (DH / 2);
#pragma unroll
        for (int j = 0; j < NJ; ++j) q[jt][j] = ld_bf16x8(qp + 8 * j);
    }
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
    const size_t row0 = ((size_t)s * a.Hkv + kvh) * a.cap;

    for (int t = t0 + wave; t < t1; t += 4) {
        const int k0 = t * kTileKeys;
        Raw<DH> raw = load_tile<DH>(a, row0, k0, lane);
        // scores
        floatx16 st[JT];
#pragma unroll
        for (int jt = 0; jt < JT; ++jt) st[jt] = floatx16{};
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const uint4 w = raw.k[j / 4];
            const uint32_t x = (j & 3) == 0 ? w.x : (j & 3) == 1 ? w.y : (j & 3) == 2 ? w.z : w.w;
            const float f = mx_scale_f((raw.ks >> (8 * (j / 4))) & 255u);
            const bf16x8 kf = as_bf16x8(fp4x2_to_bf16x2<0>(x, f), fp4x2_to_bf16x2<1>(x, f), fp4x2_to_bf16x2<2>(x, f),
                                        fp4x2_to_bf16x2<3>(x, f));
#pragma unroll
            for (int jt = 0; jt < JT; ++jt) st[jt] = mfma32x32x16(kf, q[jt][j], st[jt]);
        }
        // visibility: element 8 m + e of a lane is key k0 + 16 m + 8 eta + e
        const bool edge = k0 + kTileKeys > P;
        uint32_t seen[JT];
        uint32_t bad[NT];   // keys whose V block of 32 dims reads as NaN (edge tiles only)
        if (edge) {
            const int j0 = k0 - P;
#pragma unroll
            for (int jt = 0; jt < JT; ++jt) {
                const uint32_t* v = vis[32 * jt + lr];
                uint32_t bits;
                if (j0 < 0) {
                    bits = (v[0] << -j0) | ((1u << -j0) - 1u);   // (-j0 < 32)
                } else {
                    const int w = j0 >> 5, sh = j0 & 31;
                    bits = sh ? (v[w] >> sh) | (v[w + 1] << (32 - sh)) : v[w];
                }
                seen[jt] = bits;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    st[jt][e] = (bits >> (16 * (e / 8) + 8 * eta + e % 8)) & 1u ? st[jt][e] : -INFINITY;
            }
            // a V block with a NaN scale would reach rows that do not see its key (0 * NaN):
            // read it as zeros and note the key
            uint32_t mine = 0;
#pragma unroll
            for (int mm = 0; mm < 2; ++mm) {
                uint32_t* sc = &raw.vs[mm].x;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t b = (sc[e / 4] >> (8 * (e & 3))) & 255u;
                    if (b == 255u) {
                        mine |= 1u << (16 * mm + 8 * eta + e);
                        sc[e / 4] &= ~(255u << (8 * (e & 3)));
                    }
                }
            }
#pragma unroll
            for (int b = 0; b < NT; ++b) {
                const int src = b * (32 / NT);
                bad[b] = (uint32_t)__shfl((int)mine, src, 64) | (uint32_t)__shfl((int)mine, src + 32, 64);
            }
        }
        // softmax
        uint32_t p[JT][8];
#pragma unroll
        for (int jt = 0; jt < JT; ++jt) {
            float top = st[jt][0];
#pragma unroll
            for (int e = 1; e < 16; ++e) top = fmaxf(top, st[jt][e]);
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float mn = fmaxf(m[jt], top * c);
            const float al = exp2_fast(m[jt] - mn);
            m[jt] = mn;
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float p0 = exp2_fast(fmaf(st[jt][2 * e], c, -mn)), p1 = exp2_fast(fmaf(st[jt][2 * e + 1], c, -mn));
                sum += p0 + p1;
                p[jt][e] = pack_bf16(p0, p1);
            }
            l[jt] = l[jt] * al + sum;
#pragma unroll
            for (int t2 = 0; t2 < NT; ++t2)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[jt][t2][e] *= al;
        }
        // values
#pragma unroll
        for (int mm = 0; mm < 2; ++mm) {
            uint32_t vf[NT][4];
            const uint32_t rv[4] = {raw.v[mm].x, raw.v[mm].y, raw.v[mm].z, raw.v[mm].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {   // keys 2 i, 2 i + 1
                const uint32_t sc = i < 2 ? raw.vs[mm].x : raw.vs[mm].y;
                const float f0 = mx_scale_f((sc >> (16 * (i & 1))) & 255u), f1 = mx_scale_f((sc >> (16 * (i & 1) + 8)) & 255u);
                if constexpr (DH == 128) {
                    const uint32_t a0 = fp4x2_to_bf16x2<0>(rv[i], f0), a1 = fp4x2_to_bf16x2<1>(rv[i], f0);
                    const uint32_t b0 = fp4x2_to_bf16x2<2>(rv[i], f1), b1 = fp4x2_to_bf16x2<3>(rv[i], f1);
                    vf[0][i] = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
                    vf[1][i] = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
                    vf[2][i] = __builtin_amdgcn_perm(b1, a1, 0x05040100u);
                    vf[3][i] = __builtin_amdgcn_perm(b1, a1, 0x07060302u);
                } else {
                    const uint32_t x = rv[i] >> (8 * (lr & 1));   // this lane's two dims of the four
                    const uint32_t a0 = fp4x2_to_bf16x2<0>(x, f0), b0 = fp4x2_to_bf16x2<2>(x, f1);
                    vf[0][i] = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
                    vf[1][i] = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
                }
            }
#pragma unroll
            for (int jt = 0; jt < JT; ++jt) {
                const bf16x8 pf = as_bf16x8(p[jt][4 * mm], p[jt][4 * mm + 1], p[jt][4 * mm + 2], p[jt][4 * mm + 3]);
#pragma unroll
                for (int t2 = 0; t2 < NT; ++t2)
                    o[jt][t2] = mfma32x32x16(as_bf16x8(vf[t2][0], vf[t2][1], vf[t2][2], vf[t2][3]), pf, o[jt][t2]);
            }
        }
        if (edge) {
            // A row i = dim NT i + t: block of 32 dims (NT i + t) / 32 = i / (32 / NT), element e has i = 8 (e / 4) + ...
            uint32_t any = 0;
#pragma unroll
            for (int b = 0; b < NT; ++b) any |= bad[b];
            if (__any(any != 0)) {
#pragma unroll
                for (int jt = 0; jt < JT; ++jt)
#pragma unroll
                    for (int t2 = 0; t2 < NT; ++t2)
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (seen[jt] & bad[8 * (e / 4) * NT / 32]) o[jt][t2][e] = __uint_as_float(0x7FC00000u);
            }
        }
    }

    // merge of the four waves
#pragma unroll
    for (int jt = 0; jt < JT; ++jt) {
        l[jt] += __shfl_xor(l[jt], 32, 64);
        if (eta == 0) {
            ml[wave][jt][0][lr] = m[jt];
            ml[wave][jt][1][lr] = l[jt];
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
        for (int w = 0; w < 4; ++w) mm = fmaxf(mm, ml[w][jt][0][lr]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            f[w] = exp2_fast(ml[w][jt][0][lr] - mm);
            ll += ml[w][jt][1][lr] * f[w];
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
        if (gridDim.y == 1) {
            const float inv = 1.f / ll;
            uint32_t w[2 * NT];
#pragma unroll
            for (int i = 0; i < 2 * NT; ++i)
                w[i] = pack_bf16(r[2 * i / NT][2 * i % NT] * inv, r[(2 * i + 1) / NT][(2 * i + 1) % NT] * inv);
            uint4* dst = reinterpret_cast<uint4*>(a.out + row * DH + d0);
#pragma unroll
            for (int i = 0; i < NT / 2; ++i) dst[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        } else {
            const size_t total = (size_t)a.b * R * a.Hq, at = (size_t)blockIdx.y * total + row;
            float* dst = a.part + at * DH + d0;
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                floatx4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = r[(4 * i + e) / NT][(4 * i + e) % NT];
                *reinterpret_cast<floatx4*>(dst + 4 * i) = x;
            }
            if (wave == 0 && eta == 0) {
                float* pm = a.part + (size_t)gridDim.y * total * DH + at * 2;
                pm[0] = mm;
                pm[1] = ll;
            }
        }
    }
}

// Merge of the key splits, in split order: a thread takes 4 dims of a row.
template <int DH>
__global__ __launch_bounds__(256) void attn_mx_combine_kernel(const float* __restrict__ part, int nsplit, int64_t rows,
                                                              bf16_t* __restrict__ out) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * (DH / 4)) return;
    const int64_t row = i / (DH / 4);
    const float* ml = part + nsplit * rows * DH;
    float mm = kFloor;
    for (int s = 0; s < nsplit; ++s) mm = fmaxf(mm, ml[(s * rows + row) * 2]);
    floatx4 x = floatx4{};
    float l = 0.f;
    for (int s = 0; s < nsplit; ++s) {
        const float f = exp2_fast(ml[(s * rows + row) * 2] - mm);
        l += ml[(s * rows + row) * 2 + 1] * f;
        x += reinterpret_cast<const floatx4*>(part)[s * rows * (DH / 4) + i] * f;
    }
    const float inv = 1.f / l;
    reinterpret_cast<uint2*>(out)[i] = make_uint2(pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv));
}

struct Plan {
    int rowtiles, split, tps;
};

constexpr int kRowsPerWave = 64;

Plan plan_of(int b, int B, int Hq, int Hkv, int P) {
    Plan p;
    const int nrows = Hq / Hkv * 2 * B;
    p.rowtiles = (nrows + kRowsPerWave - 1) / kRowsPerWave;
    const int ntiles = (P + 2 * B + kTileKeys - 1) / kTileKeys;
    const int64_t wgs = (int64_t)p.rowtiles * Hkv * b;
    p.split = 1;
    if (wgs < 512) {
        p.split = (int)((512 + wgs - 1) / wgs);
        const int most = (ntiles + 7) / 8;   // two tiles a wave at least
        p.split = p.split < most ? p.split : most;
        p.split = p.split < 64 ? p.split : 64;
    }
    p.tps = (ntiles + p.split - 1) / p.split;
    p.split = (ntiles + p.tps - 1) / p.tps;
    return p;
}

}  // namespace

size_t attention_mx_partial_bytes(int b, int B, int Hq, int Hkv, int dh, int P) {
    const Plan p = plan_of(b, B, Hq, Hkv, P);
    return p.split > 1 ? (size_t)p.split * b * 2 * B * Hq * (dh + 2) * 4 : 0;
}

hipError_t launch_attention_mx(const MxAttnArgs& a, hipStream_t s) {
    const Plan p = plan_of(a.b, a.B, a.Hq, a.Hkv, a.P);
    const dim3 g((unsigned)(p.rowtiles * a.Hkv * a.b), p.split);
    if (a.dh == 128) launch(attn_mx_kernel<128, kRowsPerWave / 32>, g, dim3(256), 0, s, a, p.rowtiles, p.tps);
    else launch(attn_mx_kernel<64, kRowsPerWave / 32>, g, dim3(256), 0, s, a, p.rowtiles, p.tps);
    if (p.split > 1) {
        const int64_t rows = (int64_t)a.b * 2 * a.B * a.Hq;
        const dim3 gc((unsigned)((rows * (a.dh / 4) + 255) / 256));
        if (a.dh == 128) launch(attn_mx_combine_kernel<128>, gc, dim3(256), 0, s, a.part, p.split, rows, a.out);
        else launch(attn_mx_combine_kernel<64>, gc, dim3(256), 0, s, a.part, p.split, rows, a.out);
    }
    return hipGetLastError();
}

}  // namespace dard
