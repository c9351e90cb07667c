// attn_cache.hip -- softmax attention of new tokens over the paged cache of quantized keys and values.
//
//   a = softmax(q k^T / sqrt(dh)) v,  k_j = (ck_j - zk_j) sk_j,  v_j = (cv_j - zv_j) sv_j,
// the new token i of a sequence seeing positions 0 .. past + i.  The codes are never turned into
// values: the scores are (q . (ck_j - zk_j)) sk_j and the output sum (p_j sv_j) (cv_j - zv_j), where the
// differences are whole numbers of at most 8 bits and a sign, exact in fp16.  So both products run on the
// fp16 matrix cores (v_mfma_f32_16x16x32_f16, fp32 sums), with the queries scaled by a power of two per
// row (the largest element near 2^4) and the weights p_j sv_j by one per wave that follows the largest sv_j:
//   bf16: the queries and the weights rounded to fp16 (by at most 2^-11 relative; the output's own rounding is 2^-8),
//   fp16, fp32: each as the sum of two fp16 parts (22 bits).
//
// One wave forms S^T = K Q^T for 32 keys and 16 query rows (rows = new tokens x query heads of one key/value
// head) and O^T += V^T P^T.  The key order inside a block of 32 is chosen so that a lane's eight
// scores (two 16 x 16 tiles) are the eight keys it supplies to the second product, eight consecutive tokens:
// row m of tile t is key 8 (m / 4) + 4 t + m % 4.  No value passes between lanes in the loop: the softmax
// reference m is moved only when a score exceeds it by 2^8, and only then are maxima exchanged.
//
// Bound by HBM for few rows (the codes go from memory to registers, the next block's while one is
// used); the key axis is split over the waves of a workgroup and over workgroups, whose sums
// (m, l, O) are joined in LDS and by a second launch.
#include <algorithm>

#include "device_common.h"
#include "cache.h"

namespace jab {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LAZY = 8.f;             // log2 of what a score may exceed the reference by
constexpr int WUP = 6;                  // log2 of the weights' extra scale: p sv <= 2^(8 + 6) in fp16
constexpr int EMIN = -125;

// two codes of a word as fp16 integers, 1024 + code: bytes 0, 1 (hi false) or 2, 3
__device__ inline f16x2 biased(uint32_t w, bool hi) {
    return __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, hi ? 0x04030402u : 0x04010400u));
}
// eight codes minus their zero-points (z: 1024 + zero-point), as a matrix-core operand
__device__ inline f16x8 codes8(uint32_t w0, uint32_t w1, const f16x2 (&z)[4]) {
    const f16x2 a = biased(w0, false) - z[0], b = biased(w0, true) - z[1];
    const f16x2 c = biased(w1, false) - z[2], d = biased(w1, true) - z[3];
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ inline f16x2 both(int z) {
    const uint32_t h = 0x6400u | (uint32_t)z;
    return __builtin_bit_cast(f16x2, h | (h << 16));
}
__device__ inline f32x4 mma16(f16x8 a, f16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ inline float pow2i(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// what a lane reads of a block of 32 tokens
template <int DH, int BITS>
struct Raw {
    static constexpr int DHB = DH * BITS / 8;
    static constexpr int KB = DHB / 4 < 8 ? 8 : DHB / 4;   // key bytes of a lane and tile
    static constexpr int NV = DHB / 16 < 1 ? 1 : DHB / 16; // 16-row tiles of value bytes
    uint32_t k[2][KB / 4];
    u32x2 v[NV];
    f32x4 ks[2], vs[2];
    int kz[2];
    u32x2 vz;
    bool in;                                               // the block's page exists
};

template <int DH, int BITS>
__device__ inline void load_block(const CacheArgs &g, int s, int h, int blk, int lane, Raw<DH, BITS> &r) {
    typedef Raw<DH, BITS> R;
    const int l16 = lane & 15, grp = lane >> 4;
    const int page = __builtin_amdgcn_readfirstlane(page_of(g, s, blk * 32));
    r.in = page >= 0;
    const int64_t slot = (((int64_t)max(page, 0) * g.n_kv_heads + h) << g.page_shift) +
                         ((blk * 32) & ((1 << g.page_shift) - 1));
    const uint8_t *kb = g.k + slot * R::DHB, *vb = g.v + slot * R::DHB;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int key = 8 * (l16 >> 2) + 4 * t + (l16 & 3);
        const uint8_t *row = kb + key * R::DHB;
        if constexpr (R::KB >= 16) {
#pragma unroll
            for (int i = 0; i < R::KB / 16; ++i) {
                const u32x4 q = *reinterpret_cast<const u32x4 *>(row + 64 * i + 16 * grp);
#pragma unroll
                for (int c = 0; c < 4; ++c) r.k[t][4 * i + c] = q[c];
            }
        } else {                                           // DH 16: groups 2 and 3 meet zeros of the query
            const u32x2 q = *reinterpret_cast<const u32x2 *>(row + (R::DHB >= 32 ? 8 * grp : R::DHB >= 16 ? 8 * (grp & 1) : 0));
            r.k[t][0] = q[0];
            r.k[t][1] = q[1];
        }
        if (g.k_zero) r.kz[t] = g.k_zero[slot + key];
    }
#pragma unroll
    for (int i = 0; i < R::NV; ++i)
        r.v[i] = *reinterpret_cast<const u32x2 *>(vb + (16 * i + (R::DHB >= 16 ? l16 : l16 & 7)) * 32 + 8 * grp);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        r.ks[i] = *reinterpret_cast<const f32x4 *>(g.k_scale + slot + 8 * grp + 4 * i);
        r.vs[i] = *reinterpret_cast<const f32x4 *>(g.v_scale + slot + 8 * grp + 4 * i);
    }
    if (g.v_zero) r.vz = *reinterpret_cast<const u32x2 *>(g.v_zero + slot + 8 * grp);
}

// SPLIT: the four waves of a workgroup share 16 RT rows and deal out the key blocks; else each wave has 16 RT
// rows of its own
template <int DT, int DH, int BITS, int RT, bool SPLIT>
struct AttnCfg {
    static constexpr int NP = DT == BF16 ? 1 : 2;          // fp16 parts of queries and weights
    static constexpr int KS = DH / 32 < 1 ? 1 : DH / 32;   // steps of 32 along the head
    static constexpr int NT = DH / 16;                     // 16-row tiles of O^T
    static constexpr int ROWS = 16 * RT * (SPLIT ? 1 : 4); // rows of a workgroup
    static constexpr int QP = DH < 32 ? 40 : DH + 8;       // fp16 per row of queries in LDS (padding against conflicts)
    static constexpr size_t Q_LDS = (size_t)NP * 16 * QP * 2 * (SPLIT ? RT : 4);
    static constexpr size_t O_LDS = SPLIT ? (size_t)4 * 16 * RT * (DH + 4) * 4 : 0;
    static constexpr size_t LDS = Q_LDS > O_LDS ? Q_LDS : O_LDS;
};

template <int DT>
__device__ inline void store4(typename Mma<DT>::elem *p, f32x4 v) {
    if constexpr (DT == F32) *reinterpret_cast<f32x4 *>(p) = v;
    else *reinterpret_cast<u32x2 *>(p) = u32x2{pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3])};
}

// grid: x = (sequence, key/value head, split), y = row tiles (dealt out)
template <int DT, int DH, int BITS, int RT, bool SPLIT>
__global__ __launch_bounds__(256) void attn_cache_kernel(CacheArgs g, const void *__restrict__ yv, int64_t ldy,
                                                         void *__restrict__ av, float *__restrict__ part, int n_split) {
    typedef AttnCfg<DT, DH, BITS, RT, SPLIT> S;
    typedef typename Mma<DT>::elem elem;
    constexpr int HALF = DH / 2, QMID = (1 << (BITS - 1)) - 1;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float rowf[SPLIT ? 16 * RT : 64];           // per row: score scale (log2 units)
    __shared__ float mlE[4][16 * RT][2];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int l16 = lane & 15, grp = lane >> 4;
    const int split = blockIdx.x % n_split, sh = blockIdx.x / n_split, h = sh % g.n_kv_heads, s = sh / g.n_kv_heads;
    const SeqRows sr = seq_rows(g, s);
    const int G = g.n_heads / g.n_kv_heads;
    const int64_t n_rows = (int64_t)sr.n * G;
    const int len = (int)min((int64_t)sr.past + sr.n, (int64_t)g.cap), n_blk = (len + 31) >> 5;
    const int b0 = (int)((int64_t)n_blk * split / n_split), b1 = (int)((int64_t)n_blk * (split + 1) / n_split);

    for (int64_t tile = blockIdx.y; tile * S::ROWS < n_rows; tile += gridDim.y) {
        const int64_t row0 = tile * S::ROWS + (SPLIT ? 0 : wave * 16 * RT);     // this wave's first row
        // ---- queries: turned, scaled, split in fp16 parts, through LDS into operands
        f16x8 qf[RT][S::NP][S::KS];
        float fs[RT];                                      // the score scale of this lane's row
        int lim[RT];                                       // last position that it sees (no row: none)
        _Float16 *ql = reinterpret_cast<_Float16 *>(smem) + (SPLIT ? 0 : wave * S::NP * 16 * S::QP);
        auto prep = [&](int64_t row, int slot, int fslot, int np_stride) {      // one row by one wave
            float x0 = 0.f, x1 = 0.f;
            const bool live = lane < HALF && row < n_rows;
            const int i = live ? (int)(row / G) : 0;
            if (live) {
                const elem *q = static_cast<const elem *>(yv) + (int64_t)(sr.row + i) * ldy +
                                ((int64_t)h * G + row % G) * DH + lane;
                x0 = to_f32<DT>(q[0]);
                x1 = to_f32<DT>(q[HALF]);
            }
            uint32_t mx = max(__builtin_bit_cast(uint32_t, x0) & 0x7FFFFFFFu, __builtin_bit_cast(uint32_t, x1) & 0x7FFFFFFFu);
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) mx = max(mx, (uint32_t)__shfl_xor((int)mx, off, 64));
            const int e = min(max((int)(mx >> 23) - 127, -100), 127);           // exponent of the largest element
            const float up = pow2i(max(3 - e, -126));
            if (g.freq[0] != 0.0 && live) {
                // turns to the nearest quarter of a cycle in fp64, the rest in fp32
                const double cyc = (double)(sr.past + i) * g.freq[lane] * 0.15915494309189535;
                float sn, cs;
                sincospif((float)(2.0 * (cyc - rint(cyc))), &sn, &cs);
                const float a = x0 * up, b = x1 * up;
                x0 = a * cs - b * sn;
                x1 = b * cs + a * sn;
            } else {
                x0 *= up;
                x1 *= up;
            }
            const bool fine = mx < 0x7F800000u;
            if (lane < HALF) {
#pragma unroll
                for (int p = 0; p < S::NP; ++p) {
                    const _Float16 a = fine ? (_Float16)x0 : (_Float16)0.f, b = fine ? (_Float16)x1 : (_Float16)0.f;
                    ql[p * np_stride + slot * S::QP + lane] = a;
                    ql[p * np_stride + slot * S::QP + lane + HALF] = b;
                    x0 -= (float)a;
                    x1 -= (float)b;
                }
            }
            if constexpr (DH < 32)
                if (lane >= DH && lane < 32)
                    for (int p = 0; p < S::NP; ++p) ql[p * np_stride + slot * S::QP + lane] = (_Float16)0.f;
            // exp2 units per product unit, the power of two taken back; a row that is not finite gives NaN
            const float f = LOG2E / sqrtf((float)DH) / up;
            if (lane == 0) rowf[fslot] = fine ? f : __builtin_nanf("");
        };
        auto fetch = [&](int rt, int slot0, int np_stride) {
            // element order along the head, matching a lane's key bytes
#pragma unroll
            for (int p = 0; p < S::NP; ++p)
#pragma unroll
                for (int ks = 0; ks < S::KS; ++ks) {
                    int d;
                    if constexpr (DH == 128) d = 64 * (ks >> 1) + 16 * grp + 8 * (ks & 1);
                    else if constexpr (DH == 64) d = BITS == 8 ? 16 * grp + 8 * ks : 32 * ks + 8 * grp;
                    else d = 8 * grp;
                    qf[rt][p][ks] = *reinterpret_cast<const f16x8 *>(ql + p * np_stride + (slot0 + l16) * S::QP + d);
                }
        };
        __syncthreads();                                   // LDS of the tile before
        if constexpr (SPLIT) {
            for (int r = wave; r < 16 * RT; r += 4) prep(row0 + r, r, r, 16 * RT * S::QP);
            __syncthreads();
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                fetch(rt, 16 * rt, 16 * RT * S::QP);
                fs[rt] = rowf[16 * rt + l16];
            }
        } else {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                for (int r = 0; r < 16; ++r) prep(row0 + 16 * rt + r, r, wave * 16 + r, 16 * S::QP);
                __syncthreads();
                fetch(rt, 0, 16 * S::QP);
                fs[rt] = rowf[wave * 16 + l16];
                __syncthreads();
            }
        }
        // the first and last position that a row of the wave sees last; rows that do not exist count as the last
        int lo_lim = INT32_MAX, hi_lim = -1;
        if (row0 < n_rows) {
            lo_lim = min(sr.past + (int)(row0 / G), g.cap - 1);
            hi_lim = min(sr.past + (int)((min(row0 + 16 * RT, n_rows) - 1) / G), g.cap - 1);
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int64_t row = row0 + 16 * rt + l16;
            lim[rt] = row < n_rows ? min(sr.past + (int)(row / G), g.cap - 1) : hi_lim;
        }
        const int stride = SPLIT ? 4 : 1, first = b0 + (SPLIT ? wave : 0), end = min(b1, (hi_lim >> 5) + 1);

        float m[RT], nm[RT], l[RT];
        f32x4 o[RT][S::NT];
        int E = EMIN;
        float Rmax = pow2i(EMIN), rinv = pow2i(-EMIN);     // 2^E, 2^-E
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -__builtin_inff();
            nm[rt] = 0.f;
            l[rt] = 0.f;
#pragma unroll
            for (int t = 0; t < S::NT; ++t) o[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        auto compute = [&](const Raw<DH, BITS> &r, int blk) {
            if (!r.in) return;
            const int key0 = blk * 32 + 8 * grp;           // this lane's eight keys
            const bool edge = blk * 32 + 31 > lo_lim;
            f32x4 st[RT][2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const f16x2 z1 = both(g.k_zero ? r.kz[t] : QMID);
                const f16x2 z[4] = {z1, z1, z1, z1};
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) st[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < S::KS; ++ks) {
                    uint32_t w0, w1;
                    if constexpr (BITS == 8) {
                        w0 = r.k[t][2 * ks];
                        w1 = r.k[t][2 * ks + 1];
                    } else if constexpr (DH >= 64) {       // the first half of the steps: low nibbles
                        const int c = 2 * (ks % (S::KS / 2)), sft = ks < S::KS / 2 ? 0 : 4;
                        w0 = (r.k[t][c] >> sft) & 0x0F0F0F0Fu;
                        w1 = (r.k[t][c + 1] >> sft) & 0x0F0F0F0Fu;
                    } else {
                        const int sft = (grp & 1) * 4;
                        w0 = (r.k[t][0] >> sft) & 0x0F0F0F0Fu;
                        w1 = (r.k[t][1] >> sft) & 0x0F0F0F0Fu;
                    }
                    const f16x8 a = codes8(w0, w1, z);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int p = 0; p < S::NP; ++p) st[rt][t] = mma16(a, qf[rt][p][ks], st[rt][t]);
                }
            }
            float vs[8], big = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                vs[i] = r.vs[i >> 2][i & 3];
                if (edge) vs[i] = key0 + i <= hi_lim ? vs[i] : 0.f;             // what was never written may be anything
                big = fmaxf(big, fabsf(vs[i]));
            }
            float top[RT];
            bool move = big > Rmax;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                top[rt] = -__builtin_inff();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float t = st[rt][i >> 2][i & 3] * r.ks[i >> 2][i & 3];
                    if (edge) t = key0 + i <= lim[rt] ? t : -__builtin_inff();
                    st[rt][i >> 2][i & 3] = t;
                    top[rt] = fmaxf(top[rt], t);
                }
                move |= top[rt] * fs[rt] > m[rt] + LAZY;
            }
            if (__builtin_amdgcn_ballot_w64(move)) {       // the references move, with every sum so far
                big = fmaxf(big, __shfl_xor(big, 16, 64));
                big = fmaxf(big, __shfl_xor(big, 32, 64));
                int En = E;
                if (big > Rmax) En = min((int)(__builtin_bit_cast(uint32_t, big) >> 23) - 127 + 1, 125);
                En = __builtin_amdgcn_readfirstlane(En);
                const float down = pow2i(max(E - En, -126));
                E = En;
                Rmax = pow2i(E);
                rinv = pow2i(-E);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    float t = top[rt];
                    t = fmaxf(t, __shfl_xor(t, 16, 64));
                    t = fmaxf(t, __shfl_xor(t, 32, 64));
                    const float mn = fmaxf(m[rt], t * fs[rt]);
                    const float al = mn == m[rt] ? 1.f : exp2f(m[rt] - mn);
                    m[rt] = mn;
                    nm[rt] = mn == -__builtin_inff() ? 0.f : -mn;
                    l[rt] *= al;
                    const float f = al * down;
#pragma unroll
                    for (int t2 = 0; t2 < S::NT; ++t2)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[rt][t2][i] *= f;
                }
            }
            const float up = rinv * (float)(1 << WUP);
#pragma unroll
            for (int i = 0; i < 8; ++i) vs[i] *= up;
            f16x8 pw[RT][S::NP];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(st[rt][i >> 2][i & 3], fs[rt], nm[rt]));
                    l[rt] += p;
                    w[i] = p * vs[i];
                }
#pragma unroll
                for (int p = 0; p < S::NP; ++p)
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const f16x2 hw = __builtin_convertvector(f32x2_t{w[i], w[i + 1]}, f16x2);
                        pw[rt][p][i] = hw[0];
                        pw[rt][p][i + 1] = hw[1];
                        if (p + 1 < S::NP) {
                            w[i] -= (float)hw[0];
                            w[i + 1] -= (float)hw[1];
                        }
                    }
            }
            f16x2 z[4];
            if (g.v_zero) {
                z[0] = biased(r.vz[0], false);
                z[1] = biased(r.vz[0], true);
                z[2] = biased(r.vz[1], false);
                z[3] = biased(r.vz[1], true);
            } else {
                z[0] = z[1] = z[2] = z[3] = both(QMID);
            }
#pragma unroll
            for (int t = 0; t < S::NT; ++t) {
                uint32_t w0, w1;
                if constexpr (BITS == 8) {
                    w0 = r.v[t][0];
                    w1 = r.v[t][1];
                } else if constexpr (DH >= 64) {
                    const int c = t % (S::NT / 2), sft = t < S::NT / 2 ? 0 : 4;
                    w0 = (r.v[c][0] >> sft) & 0x0F0F0F0Fu;
                    w1 = (r.v[c][1] >> sft) & 0x0F0F0F0Fu;
                } else {
                    const int sft = (l16 >> 3) * 4;
                    w0 = (r.v[0][0] >> sft) & 0x0F0F0F0Fu;
                    w1 = (r.v[0][1] >> sft) & 0x0F0F0F0Fu;
                }
                const f16x8 a = codes8(w0, w1, z);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int p = 0; p < S::NP; ++p) o[rt][t] = mma16(a, pw[rt][p], o[rt][t]);
            }
        };
        if (first < end) {
            Raw<DH, BITS> ra, rb;
            int b = first;
            load_block(g, s, h, b, lane, ra);
            for (;;) {
                if (b + stride < end) load_block(g, s, h, b + stride, lane, rb);
                compute(ra, b);
                b += stride;
                if (b >= end) break;
                if (b + stride < end) load_block(g, s, h, b + stride, lane, ra);
                compute(rb, b);
                b += stride;
                if (b >= end) break;
            }
        }

        // ---- sums over a row's four lane groups; the weights' scale taken back
        const float back = pow2i(max(E - WUP, -126));
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            l[rt] += __shfl_xor(l[rt], 16, 64);
            l[rt] += __shfl_xor(l[rt], 32, 64);
#pragma unroll
            for (int t = 0; t < S::NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[rt][t][i] *= back;
        }
        // one row's four elements d .. d + 3: the output, or the split's share of it
        auto put = [&](int64_t row, int d, f32x4 v, float mm, float ll) {
            if (row >= n_rows) return;
            const int64_t tok = sr.row + row / G, head = (int64_t)h * G + row % G;
            if (n_split == 1) {
                const float inv = ll == 0.f ? 0.f : 1.f / ll;
                store4<DT>(static_cast<elem *>(av) + (tok * g.n_heads + head) * DH + d,
                           f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv});
            } else {
                float *pp = part + ((tok * g.n_heads + head) * n_split + split) * (DH + 4);
                *reinterpret_cast<f32x4 *>(pp + d) = v;
                if (d == 0) {
                    pp[DH] = mm;
                    pp[DH + 1] = ll;
                }
            }
        };
        if constexpr (!SPLIT) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int t = 0; t < S::NT; ++t) put(row0 + 16 * rt + l16, 16 * t + 4 * grp, o[rt][t], m[rt], l[rt]);
        } else {
            // the four waves' sums, through LDS
            float *ol = reinterpret_cast<float *>(smem);
            __syncthreads();                               // every wave has its queries
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                if (grp == 0) {
                    mlE[wave][16 * rt + l16][0] = m[rt];
                    mlE[wave][16 * rt + l16][1] = l[rt];
                }
#pragma unroll
                for (int t = 0; t < S::NT; ++t)
                    *reinterpret_cast<f32x4 *>(ol + ((wave * 16 * RT) + 16 * rt + l16) * (DH + 4) + 16 * t + 4 * grp) = o[rt][t];
            }
            __syncthreads();
            const int live = (int)min((int64_t)16 * RT, n_rows - row0);
            for (int c = threadIdx.x; c < live * (DH / 4); c += 256) {
                const int r = c / (DH / 4), d = c % (DH / 4) * 4;
                float mm = -__builtin_inff();
#pragma unroll
                for (int w = 0; w < 4; ++w) mm = fmaxf(mm, mlE[w][r][0]);
                f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
                float ll = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    // a wave without a key has m = -inf, l = 0; a NaN row keeps m = -inf and l = NaN
                    const float f = mlE[w][r][0] == mm ? 1.f : exp2f(mlE[w][r][0] - mm);
                    const f32x4 x = *reinterpret_cast<const f32x4 *>(ol + (w * 16 * RT + r) * (DH + 4) + d);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] += f * x[i];
                    ll += f * mlE[w][r][1];
                }
                put(row0 + r, d, v, mm, ll);
            }
        }
    }
}

// The splits of a row joined: one wave per (token, head) and pass, the splits over its lane groups.
// part [row][split][DH + 4]: O, m, l
template <int DT, int DH>
__global__ __launch_bounds__(256) void attn_join_kernel(CacheArgs g, const float *__restrict__ part, void *__restrict__ av,
                                                        int n_split) {
    typedef typename Mma<DT>::elem elem;
    constexpr int LPR = DH / 4, SG = 64 / LPR;             // lanes of a row, splits at once
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int s = blockIdx.x;
    const SeqRows sr = seq_rows(g, s);
    const int64_t items = (int64_t)sr.n * g.n_heads;
    const int d = lane % LPR * 4, sg = lane / LPR;
    for (int64_t it = (int64_t)blockIdx.y * 4 + wave; it < items; it += (int64_t)gridDim.y * 4) {
        const int64_t row = (int64_t)sr.row * g.n_heads + it;
        const float *p = part + row * n_split * (DH + 4);
        float m = -__builtin_inff();
        for (int i = lane; i < n_split; i += 64) m = fmaxf(m, p[(int64_t)i * (DH + 4) + DH]);
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
        f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
#pragma unroll 4
        for (int i = sg; i < n_split; i += SG) {
            const float *q = p + (int64_t)i * (DH + 4);
            const float mi = q[DH], f = mi == m ? 1.f : exp2f(mi - m);
            const f32x4 x = *reinterpret_cast<const f32x4 *>(q + d);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += f * x[k];
            l += f * q[DH + 1];
        }
#pragma unroll
        for (int off = 32; off >= LPR; off >>= 1) {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += __shfl_xor(v[k], off, 64);
            l += __shfl_xor(l, off, 64);
        }
        if (sg == 0) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            store4<DT>(static_cast<elem *>(av) + row * DH + d, f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv});
        }
    }
}

constexpr int CUS = 256;
// Rows of one key/value head, the wave arrangement and the splits of the key axis.
struct Plan {
    bool split_waves;                   // the waves of a workgroup share their rows
    int rt;                             // 16-row tiles per wave
    int n_split;
    int64_t tiles;                      // workgroup row tiles per (sequence, head)
};
Plan plan_of(const CacheArgs &g) {
    Plan p;
    const int64_t rows = (int64_t)std::max(g.max_new, 1) * (g.n_heads / g.n_kv_heads);
    p.split_waves = rows <= 32;
    p.rt = rows <= 16 ? 1 : 2;
    const int per = 16 * p.rt * (p.split_waves ? 1 : 4);
    p.tiles = (rows + per - 1) / per;
    // enough workgroups for every CU to hold several, each with at least 8 blocks of 32 keys
    const int64_t base = (int64_t)g.n_seq * g.n_kv_heads * p.tiles, blocks = ((int64_t)g.cap + 31) / 32;
    const int64_t want = (4 * CUS + base - 1) / base, most = std::max<int64_t>(1, blocks / 8);
    p.n_split = (int)std::min<int64_t>(std::min(want, most), 128);
    return p;
}

template <int DT, int DH, int BITS, int RT, bool SPLIT>
hipError_t run_attn(const CacheArgs &g, const Plan &p, const void *y, int64_t ldy, void *a, float *part, hipStream_t st) {
    typedef AttnCfg<DT, DH, BITS, RT, SPLIT> S;
    hipError_t e = hipFuncSetAttribute((const void *)attn_cache_kernel<DT, DH, BITS, RT, SPLIT>,
                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)S::LDS);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)(g.n_seq * g.n_kv_heads * p.n_split), (unsigned)std::min<int64_t>(p.tiles, 65535));
    attn_cache_kernel<DT, DH, BITS, RT, SPLIT><<<grid, 256, S::LDS, st>>>(g, y, ldy, a, part, p.n_split);
    e = hipGetLastError();
    if (e != hipSuccess || p.n_split == 1) return e;
    const int64_t items = (int64_t)std::max(g.max_new, 1) * g.n_heads;
    attn_join_kernel<DT, DH><<<dim3(g.n_seq, (unsigned)std::min<int64_t>((items + 3) / 4, 65535)), 256, 0, st>>>(g, part, a, p.n_split);
    return hipGetLastError();
}

template <int DT, int DH, int BITS>
hipError_t run_plan(const CacheArgs &g, const void *y, int64_t ldy, void *a, void *ws, hipStream_t st) {
    const Plan p = plan_of(g);
    float *part = static_cast<float *>(ws);
    if (!p.split_waves) return run_attn<DT, DH, BITS, 2, false>(g, p, y, ldy, a, part, st);
    return p.rt == 1 ? run_attn<DT, DH, BITS, 1, true>(g, p, y, ldy, a, part, st)
                     : run_attn<DT, DH, BITS, 2, true>(g, p, y, ldy, a, part, st);
}
template <int DT, int DH>
hipError_t run_bits(const CacheArgs &g, const void *y, int64_t ldy, void *a, void *ws, hipStream_t st) {
    return g.bits == 8 ? run_plan<DT, DH, 8>(g, y, ldy, a, ws, st) : run_plan<DT, DH, 4>(g, y, ldy, a, ws, st);
}
template <int DT>
hipError_t run_dh(const CacheArgs &g, const void *y, int64_t ldy, void *a, void *ws, hipStream_t st) {
    switch (g.head_dim) {
    case 16: return run_bits<DT, 16>(g, y, ldy, a, ws, st);
    case 64: return run_bits<DT, 64>(g, y, ldy, a, ws, st);
    default: return run_bits<DT, 128>(g, y, ldy, a, ws, st);
    }
}
}  // namespace

size_t attn_cache_ws_bytes(const CacheArgs &g) {
    const Plan p = plan_of(g);
    return p.n_split == 1 ? 0 : (size_t)g.M * g.n_heads * p.n_split * (g.head_dim + 4) * sizeof(float);
}

hipError_t launch_attn_cache(int dtype, const CacheArgs &g, const void *y, int64_t ldy, void *a, void *ws, hipStream_t st) {
    switch (dtype) {
    case F32: return run_dh<F32>(g, y, ldy, a, ws, st);
    case F16: return run_dh<F16>(g, y, ldy, a, ws, st);
    default: return run_dh<BF16>(g, y, ldy, a, ws, st);
    }
}

}  // namespace jab
