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
constexpr int EMIN = -119;              // 2^(WUP - EMIN) is finite
constexpr int NOWHERE = INT32_MAX - 63; // a key past every position

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

// The bytes of a block of 32 tokens that one lane supplies to the products, eight consecutive ones at a time
// ("units"): a unit is one operand at 8 bits, two at 4 bits (low and high halves), half of one at head_dim 16.
template <int DH, int BITS>
struct Lay {
    static constexpr int DHB = DH * BITS / 8;
    static constexpr int KS = DH / 32 < 1 ? 1 : DH / 32;                 // steps of 32 along the head
    static constexpr int NT = DH / 16;                                   // 16-row tiles of O^T
    static constexpr int KU = DH < 64 ? 1 : KS * BITS / 8;               // key units of a 16-key tile
    static constexpr int VU = DH < 64 ? 1 : NT * BITS / 8;               // value units
    // key row m of tile t
    static __device__ inline int key(int t, int l16) { return 8 * (l16 >> 2) + 4 * t + (l16 & 3); }
    // byte of key unit u in its row; groups 2 and 3 of head_dim 16 meet zeros of the query
    static __device__ inline int kbyte(int u, int grp) {
        if constexpr (DHB >= 64) return 64 * (u >> 1) + 16 * grp + 8 * (u & 1);
        else if constexpr (DHB == 32) return 8 * grp;
        else if constexpr (DHB == 16) return 8 * (grp & 1);
        else return 0;
    }
    // byte row of value unit u
    static __device__ inline int vrow(int u, int l16) { return 16 * u + (DHB >= 16 ? l16 : l16 & 7); }
    // first element along the head of step ks (the query's order)
    static __device__ inline int dim(int ks, int grp) {
        if constexpr (DH == 128) return 64 * (ks >> 1) + 16 * grp + 8 * (ks & 1);
        else if constexpr (DH == 64) return BITS == 8 ? 16 * grp + 8 * ks : 32 * ks + 8 * grp;
        else return 8 * grp;
    }
    // the operand of step ks (tile t) from the units' bytes
    static __device__ inline f16x8 kop(const u32x2 (&k)[KU], int ks, int grp, const f16x2 (&z)[4]) {
        if constexpr (BITS == 8) return codes8(k[ks][0], k[ks][1], z);
        else {
            const int u = DH < 64 ? 0 : ks % KU, sft = DH < 64 ? (grp & 1) * 4 : ks < KU ? 0 : 4;
            return codes8((k[u][0] >> sft) & 0x0F0F0F0Fu, (k[u][1] >> sft) & 0x0F0F0F0Fu, z);
        }
    }
    static __device__ inline f16x8 vop(const u32x2 (&v)[VU], int t, int l16, const f16x2 (&z)[4]) {
        if constexpr (BITS == 8) return codes8(v[t][0], v[t][1], z);
        else {
            const int u = DH < 64 ? 0 : t % VU, sft = DH < 64 ? (l16 >> 3) * 4 : t < VU ? 0 : 4;
            return codes8((v[u][0] >> sft) & 0x0F0F0F0Fu, (v[u][1] >> sft) & 0x0F0F0F0Fu, z);
        }
    }
};

// from a wave-uniform base and a lane's byte offset
template <typename T>
__device__ inline T ldu(const uint8_t *base, uint32_t off) {
    asm("" : "+v"(off));                                   // widened at the load: else kept widened, twice the registers
    return *reinterpret_cast<const T *>(base + off);
}
// the same of bytes that one workgroup reads, once: few rows 64 x 8 heads 103 us instead of 107, one of 130000 tokens 37
// instead of 38.5 (many rows, whose blocks several workgroups read, 664 instead of 600)
template <typename T>
__device__ inline T ldu_once(const uint8_t *base, uint32_t off) {
    return __builtin_nontemporal_load(reinterpret_cast<const T *>(base + off));
}

// where block blk of a sequence lies: its first slot, or -1
__device__ inline int64_t block_slot(const CacheArgs &g, int s, int h, int blk) {
    const int page = __builtin_amdgcn_readfirstlane(page_of(g, s, blk * 32));
    if (page < 0) return -1;
    return (((int64_t)page * g.n_kv_heads + h) << g.page_shift) + ((blk * 32) & ((1 << g.page_shift) - 1));
}

// The softmax state of 16 RT rows of one wave: lane (l16, grp) holds row l16 of each tile, of O^T its elements
// 16 t + 4 grp .. + 3, of l the part of its own keys.
template <int DT, int DH, int BITS, int RT>
struct Wave {
    static constexpr int NP = DT == BF16 ? 1 : 2;          // fp16 parts of queries and weights
    typedef Lay<DH, BITS> L;
    f16x8 qf[RT][NP][L::KS];
    float fs[RT];                                          // score scale (exp2 units)
    int lim[RT], lo_lim, hi_lim;                           // last position seen: by this lane's rows, least and most of the wave
    float m[RT], nm[RT], l[RT];
    f32x4 o[RT][L::NT];
    int E;
    float Rmax, rinv;                                      // 2^E, 2^-E

    __device__ inline void limits(const CacheArgs &g, const SeqRows &sr, int G, int row0, int n_rows, int l16) {
        lo_lim = INT32_MAX;
        hi_lim = -1;
        if (row0 < n_rows) {
            lo_lim = min(sr.past + row0 / G, g.cap - 1);
            hi_lim = min(sr.past + (min(row0 + 16 * RT, n_rows) - 1) / G, g.cap - 1);
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {                  // rows that do not exist count as the last
            const int row = row0 + 16 * rt + l16;
            lim[rt] = row < n_rows ? min(sr.past + row / G, g.cap - 1) : hi_lim;
        }
    }
    __device__ inline void start() {
        E = EMIN;
        Rmax = pow2i(EMIN);
        rinv = pow2i(-EMIN);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -__builtin_inff();
            nm[rt] = 0.f;
            l[rt] = 0.f;
#pragma unroll
            for (int t = 0; t < L::NT; ++t) o[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    // S^T of a block, kop(t, ks) the key operands (few at a time in registers)
    template <typename F>
    __device__ inline void scores(f32x4 (&st)[RT][2], F &&kop) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) st[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < L::KS; ++ks) {
                const f16x8 a = kop(t, ks);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int p = 0; p < NP; ++p) st[rt][t] = mma16(a, qf[rt][p][ks], st[rt][t]);
                if (ks & 1) __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    // the scores in key units: times the keys' scales; -inf where not seen (key0: this lane's first key)
    __device__ inline void scale(f32x4 (&st)[RT][2], const f32x4 (&ks)[2]) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int i = 0; i < 8; ++i) st[rt][i >> 2][i & 3] *= ks[i >> 2][i & 3];
    }
    __device__ inline void mask(f32x4 (&st)[RT][2], bool edge, int key0) {
        if (edge) {
            asm volatile("");                              // a branch, so that other blocks pay nothing for the masks
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    st[rt][i >> 2][i & 3] = key0 + i <= lim[rt] ? st[rt][i >> 2][i & 3] : -__builtin_inff();
        }
    }
    // A block's value scales.  In a block that not every row sees whole, what was never written (or has no page) may be
    // anything and counts 0; and a value that is NaN goes over to the scores of the rows that see it, since its
    // product with the weight 0 of the others would be NaN too.
    __device__ inline void value_scales(f32x4 (&st)[RT][2], const f32x4 (&vsc)[2], bool edge, int key0, float (&vs)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) vs[i] = vsc[i >> 2][i & 3];
        if (edge) {
            asm volatile("");
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = key0 + i <= hi_lim, fine = fabsf(vs[i]) < __builtin_inff();
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const float t = st[rt][i >> 2][i & 3];
                    st[rt][i >> 2][i & 3] = fine || t == -__builtin_inff() ? t : __builtin_nanf("");
                }
                vs[i] = in && fine ? vs[i] : 0.f;
            }
        }
    }
    // the references moved where a block's scores or value scales ask for it, with every sum so far
    __device__ inline void move(const f32x4 (&st)[RT][2], const float (&vs)[8]) {
        float big = 0.f, top[RT];
#pragma unroll
        for (int i = 0; i < 8; ++i) big = fmaxf(big, fabsf(vs[i]));
        bool any = big > Rmax;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            top[rt] = st[rt][0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top[rt] = fmaxf(top[rt], st[rt][i >> 2][i & 3]);
            any |= top[rt] * fs[rt] > m[rt] + LAZY;
        }
        if (!__builtin_amdgcn_ballot_w64(any)) return;
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
            for (int t2 = 0; t2 < L::NT; ++t2)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[rt][t2][i] *= f;
        }
    }
    // the weights of two scores of a lane: piece j = 4 rt + k, keys 2 k and 2 k + 1; vs: the value scales times up()
    __device__ inline float up() const { return rinv * (float)(1 << WUP); }
    __device__ inline void weight2(int j, const f32x4 (&st)[RT][2], const float (&vs)[8], f16x8 (&pw)[RT][NP]) {
        const int rt = j >> 2, i = 2 * (j & 3);
        float w[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(st[rt][i >> 2][(i & 3) + e], fs[rt], nm[rt]));
            l[rt] += p;
            w[e] = p * vs[i + e];
        }
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const f16x2 hw = __builtin_convertvector(f32x2_t{w[0], w[1]}, f16x2);
            pw[rt][p][i] = hw[0];
            pw[rt][p][i + 1] = hw[1];
            if (p + 1 < NP) {
                w[0] -= (float)hw[0];
                w[1] -= (float)hw[1];
            }
        }
    }
    // O^T += V^T P^T, vop(t) the value operands
    template <typename F>
    __device__ inline void values(const f16x8 (&pw)[RT][NP], F &&vop) {
#pragma unroll
        for (int t = 0; t < L::NT; ++t) {
            const f16x8 a = vop(t);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int p = 0; p < NP; ++p) o[rt][t] = mma16(a, pw[rt][p], o[rt][t]);
            if (t & 1) __builtin_amdgcn_sched_barrier(0);
        }
    }
    // sums over a row's four lane groups; the weights' scale taken back
    __device__ inline void finish() {
        const float back = pow2i(max(E - WUP, -126));
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            l[rt] += __shfl_xor(l[rt], 16, 64);
            l[rt] += __shfl_xor(l[rt], 32, 64);
#pragma unroll
            for (int t = 0; t < L::NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[rt][t][i] *= back;
        }
    }
};

// Queries in LDS: QP fp16 per row (padding against bank conflicts), the parts `stride` apart
template <int DH> constexpr int QP = DH < 32 ? 40 : DH + 8;

// the power of two that brings a row whose largest magnitude has the bits mx near 2^4
__device__ inline float query_scale(uint32_t mx) {
    const int e = min(max((int)(mx >> 23) - 127, -100), 127);
    return pow2i(max(3 - e, -126));
}
// the pair (a, b) turned at a position: whole cycles are taken off the angle in fp64, the rest is fp32
__device__ inline void turn(float &a, float &b, int pos, double freq) {
    const double cyc = (double)pos * freq * 0.15915494309189535;
    float sn, cs;
    sincospif((float)(2.0 * (cyc - rint(cyc))), &sn, &cs);
    const float x = a, y = b;
    a = x * cs - y * sn;
    b = y * cs + x * sn;
}
// a pair's fp16 parts at ql and ql + half, the next part `stride` on
template <int NP>
__device__ inline void query_parts(float a, float b, _Float16 *ql, int half, int stride) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const _Float16 ha = (_Float16)a, hb = (_Float16)b;
        ql[p * stride] = ha;
        ql[p * stride + half] = hb;
        a -= (float)ha;
        b -= (float)hb;
    }
}

// One query row by one wave: turned, scaled by a power of two, as fp16 parts into row `slot` of ql; returns the
// score scale in exp2 units with the power of two taken back (NaN for a row that is not finite)
template <int DT, int DH, int NP>
__device__ inline float query_row(const CacheArgs &g, const SeqRows &sr, const void *yv, int64_t ldy, int h, int G, int row,
                                  _Float16 *ql, int slot, int stride, int lane) {
    typedef typename Mma<DT>::elem elem;
    constexpr int HALF = DH / 2;
    float x0 = 0.f, x1 = 0.f;
    const int i = row / G;
    if (lane < HALF) {
        const elem *q = static_cast<const elem *>(yv) + (int64_t)(sr.row + i) * ldy + ((int64_t)h * G + row % G) * DH + lane;
        x0 = to_f32<DT>(q[0]);
        x1 = to_f32<DT>(q[HALF]);
    }
    uint32_t mx = max(__builtin_bit_cast(uint32_t, x0) & 0x7FFFFFFFu, __builtin_bit_cast(uint32_t, x1) & 0x7FFFFFFFu);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) mx = max(mx, (uint32_t)__shfl_xor((int)mx, off, 64));
    const float up = query_scale(mx);
    x0 *= up;
    x1 *= up;
    if (g.freq[0] != 0.0 && lane < HALF) turn(x0, x1, sr.past + i, g.freq[lane]);
    const bool fine = mx < 0x7F800000u;
    _Float16 *q = ql + slot * QP<DH> + lane;
    if (lane < HALF) query_parts<NP>(fine ? x0 : 0.f, fine ? x1 : 0.f, q, HALF, stride);
    if constexpr (DH < 32)
        if (lane >= DH && lane < 32 - HALF) query_parts<NP>(0.f, 0.f, q, HALF, stride);
    return fine ? LOG2E / sqrtf((float)DH) / up : __builtin_nanf("");
}

// The same for sixteen rows row0 .. of one wave, sixteen lanes per row, into rows 0 .. 15 of ql and rowf
template <int DT, int DH, int NP>
__device__ inline void query_rows16(const CacheArgs &g, const SeqRows &sr, const void *yv, int64_t ldy, int h, int G, int row0,
                                    int n_rows, _Float16 *ql, int stride, float *rowf, int lane) {
    typedef typename Mma<DT>::elem elem;
    constexpr int HALF = DH / 2, C = HALF / 16 < 1 ? 1 : HALF / 16;             // pairs of a lane
    const int j0 = (lane & 15) * C;
    const bool in = j0 < HALF;                             // head_dim 16: eight lanes per row
    float x[4][2][C];
    int tok[4];
    bool live[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {                          // all loads first
        const int row = row0 + 4 * i + (lane >> 4);
        live[i] = row < n_rows && in;
        tok[i] = live[i] ? row / G : 0;
        const elem *q = static_cast<const elem *>(yv) + (int64_t)(sr.row + tok[i]) * ldy + ((int64_t)h * G + (live[i] ? row % G : 0)) * DH +
                        (in ? j0 : 0);
        elem e[2][C];
        __builtin_memcpy(e[0], __builtin_assume_aligned(q, C * sizeof(elem)), C * sizeof(elem));
        __builtin_memcpy(e[1], __builtin_assume_aligned(q + HALF, C * sizeof(elem)), C * sizeof(elem));
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int c = 0; c < C; ++c) x[i][u][c] = live[i] ? to_f32<DT>(e[u][c]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t mx = 0;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int c = 0; c < C; ++c) mx = max(mx, __builtin_bit_cast(uint32_t, x[i][u][c]) & 0x7FFFFFFFu);
        mx = max(mx, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)mx, 0x128, 0xF, 0xF, false));    // row_ror 8, 4, 2, 1
        mx = max(mx, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)mx, 0x124, 0xF, 0xF, false));
        mx = max(mx, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)mx, 0x122, 0xF, 0xF, false));
        mx = max(mx, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)mx, 0x121, 0xF, 0xF, false));
        const float up = query_scale(mx);
        const bool fine = mx < 0x7F800000u;
        const int slot = 4 * i + (lane >> 4);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float a = x[i][0][c] * up, b = x[i][1][c] * up;
            if (g.freq[0] != 0.0) turn(a, b, sr.past + tok[i], g.freq[in ? j0 + c : 0]);
            if (in)
                query_parts<NP>(fine ? a : 0.f, fine ? b : 0.f, ql + slot * QP<DH> + j0 + c, HALF, stride);
            else if constexpr (DH < 32) {                  // zeros behind the head: the step is 32 elements
                query_parts<NP>(0.f, 0.f, ql + slot * QP<DH> + 16 + j0 - HALF, HALF, stride);
            }
        }
        if ((lane & 15) == 0) rowf[slot] = fine ? LOG2E / sqrtf((float)DH) / up : __builtin_nanf("");
    }
}

template <int DT>
__device__ inline void store4(typename Mma<DT>::elem *p, f32x4 v) {
    if constexpr (DT == F32) *reinterpret_cast<f32x4 *>(p) = v;
    else *reinterpret_cast<u32x2 *>(p) = u32x2{pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3])};
}
// ---------------------------------------------------------------- shares
// The work is a list of blocks of 32 keys: for each key/value head, sequence and tile of ROWS query rows, the blocks
// up to the last position that the tile sees.  It is cut in equal shares, one per workgroup, wherever the
// sequences' lengths put the cuts (only the device knows them), so no workgroup is left with a long sequence.
// A cut closer than SNAP blocks to a tile's end moves there.  A tile that lies in one share is written as output;
// a share has at most two pieces of others, its first (slot 0: the tile began in an earlier share) and its last (slot 1:
// the tile begins here), which attn_join_kernel joins.
constexpr int SNAP = 8, SHARE = 8;      // least blocks of a piece, of a share (4 for either or both: 1 x 940 rows on 34892
                                        // keys 194 .. 223 us for 203, 2 x 2048 on 512 43 .. 53 for 50, 8 x 512 on 528 42 .. 50
                                        // for 39, single tokens the same)
constexpr int SCAN_SEQS = 512;          // sequences up to which each workgroup scans them; past it one workgroup per
                                        // (sequence, head), of which there are then enough (1024 x 8 of 1600 tokens: 581 us,
                                        // 634 with shares; 512: 285 and 313, but uneven lengths want them)
// Blocks, over all tiles of a (sequence, head), below which it goes to one workgroup: shares cost their scan and the
// join's launch.  One new token, whole / shares: 800 tokens 12.4 / 13.9 us, 1500 17.2 / 16.1, 6000 50 / 15; 16 sequences
// 14.7 / 20.5, 25.2 / 25.4, 84 / 48.  128 rows on 432 tokens 25.0 / 28.0, on 832 36.6 / 25.7; 2048 rows on 512 268 / 49.
constexpr int WHOLE_FEW = 48, WHOLE_MANY = 20;

template <int ROWS>
__device__ inline int tile_blocks(const CacheArgs &g, const SeqRows &r, int G, int tile) {
    const int end = (tile + 1) * ROWS, tok = end >= r.n * G ? r.n - 1 : (end - 1) / G;
    return (min(r.past + tok, g.cap - 1) >> 5) + 1;
}
// blocks of one head of a sequence
template <int ROWS>
__device__ inline uint32_t head_blocks(const CacheArgs &g, const SeqRows &r, int G) {
    uint32_t sum = 0;
    for (int t = 0; t * ROWS < r.n * G; ++t) sum += tile_blocks<ROWS>(g, r, G, t);
    return sum;
}
// inclusive sum over the wave's lanes: rows of 16 by shifts, then the rows before
__device__ inline uint32_t wave_scan(uint32_t v) {
    auto add = [&](auto ctrl, auto rows) {
        v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
    };
    typedef std::integral_constant<int, 0xF> all;
    add(std::integral_constant<int, 0x111>(), all());      // row_shr 1, 2, 4, 8
    add(std::integral_constant<int, 0x112>(), all());
    add(std::integral_constant<int, 0x114>(), all());
    add(std::integral_constant<int, 0x118>(), all());
    add(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xA>());      // row_bcast 15 into rows 1, 3
    add(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xC>());      // row_bcast 31 into rows 2, 3
    return v;
}
__device__ inline uint32_t lane_value(uint32_t v, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); }

struct Piece {                          // what a slot holds
    int s, h, tile;
    int flag;                           // 0 nothing, 1 a part, 2 the part that ends the tile
};

// The workgroup's share: where it starts and its blocks (wave-uniform; a head's blocks of all sequences stay below
// 2^31).  SCAN: equal shares; else a (sequence, head) per workgroup.
template <int ROWS, bool SCAN>
struct Share {
    int s, h, tile, blk;
    int64_t left;

    __device__ inline void advance(const CacheArgs &g, int G) {        // to the start of the next tile
        blk = 0;
        if (++tile * ROWS < seq_rows(g, s).n * G) return;
        tile = 0;
#pragma unroll 1
        for (int k = 0; k <= g.n_seq; ++k) {               // the next sequence with new tokens, or the next head's first
            if (++s == g.n_seq) {
                s = 0;
                ++h;
            }
            if (seq_rows(g, s).n > 0) return;
        }
    }
    __device__ inline void find(const CacheArgs &g, int G, int share, int n_shares, int lane) {
        left = 0;
        if constexpr (!SCAN) {
            s = share / g.n_kv_heads;
            h = share - s * g.n_kv_heads;
            tile = blk = 0;
            const SeqRows r = seq_rows(g, s);
#pragma unroll 1
            for (int t = 0; t * ROWS < r.n * G; ++t) left += tile_blocks<ROWS>(g, r, G, t);
            return;
        }
        // lane i: the blocks of sequences i per .. (i + 1) per - 1
        const int per = (g.n_seq + 63) / 64;
        uint32_t sum = 0;
#pragma unroll 1
        for (int i = lane * per; i < min((lane + 1) * per, g.n_seq); ++i) sum += head_blocks<ROWS>(g, seq_rows(g, i), G);
        const uint32_t inc = wave_scan(sum), total = lane_value(inc, 63);
        if (total == 0) return;
        const int n = (int)min((int64_t)n_shares, max((int64_t)total * g.n_kv_heads / SHARE, (int64_t)1));
        if (share >= n) return;
        const double step = (double)total / n;             // a cut is the same number for the shares on both its sides
        int64_t to = 0;
#pragma unroll 1
        for (int e = 1; e >= 0; --e) {                     // where the share ends, then where it starts
            const uint32_t u = (uint32_t)(share + e) * (uint32_t)g.n_kv_heads;
            h = (int)(u / (uint32_t)n);
            uint32_t x = min((uint32_t)((double)(u - (uint32_t)h * n) * step), total - 1);
            int64_t at = (int64_t)h * total + x;
            s = tile = blk = 0;
            if (h < g.n_kv_heads) {
                const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(inc > x));
                x -= l ? lane_value(inc, l - 1) : 0u;
                s = l * per;
                SeqRows r = seq_rows(g, s);
                uint32_t nb = r.n > 0 ? tile_blocks<ROWS>(g, r, G, 0) : 0;
                const int stop = min((l + 1) * per, g.n_seq) - 1;
#pragma unroll 1
                while (x >= nb) {                          // the next tile, of the lane's next sequence after the last one
                    x -= nb;
                    if (++tile * ROWS >= r.n * G) {
                        if (s == stop) break;              // (never, unless the tables change under the call)
                        tile = 0;
                        r = seq_rows(g, ++s);
                    }
                    nb = r.n > 0 ? tile_blocks<ROWS>(g, r, G, tile) : 0;
                }
                blk = (int)x;
                if (blk < SNAP) {
                    at -= blk;
                    blk = 0;
                } else if ((int)nb - blk < SNAP) {
                    at += (int)nb - blk;
                    advance(g, G);
                }
            }
            if (e) to = at;
            else left = to - at;
        }
    }
};

// workgroup -> share: an XCD (ids congruent mod 8) takes a contiguous range, so that tiles that read the same keys share
// its L2
__device__ inline int share_of(int block, int n_shares) {
    return (n_shares & 7) == 0 ? (block & 7) * (n_shares >> 3) + (block >> 3) : block;
}

// four elements d .. d + 3 of a row: the output, or (part: the slot's rows, [row][DH + 4]: O, m, l) a piece of it
template <int DT, int DH>
__device__ inline void put_row(const CacheArgs &g, const SeqRows &sr, int h, int G, int row0, int r, int d, f32x4 v, float m, float l,
                               void *av, float *part) {
    typedef typename Mma<DT>::elem elem;
    if (part == nullptr) {
        const int row = row0 + r;
        const int64_t at = (int64_t)(sr.row + row / G) * g.n_heads + (int64_t)h * G + row % G;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        store4<DT>(static_cast<elem *>(av) + at * DH + d, f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv});
    } else {
        float *pp = part + r * (DH + 4);
        *reinterpret_cast<f32x4 *>(pp + d) = v;
        if (d == 0) {
            pp[DH] = m;
            pp[DH + 1] = l;
        }
    }
}

// ---------------------------------------------------------------- few rows
// The four waves of a workgroup share 16 RT rows and deal out the key blocks.  Codes go from memory to
// registers; a block's keys are asked for once the previous block's scores are formed, its values once the
// previous block's are used, so one block is in flight per wave without a second set of registers.
// Measured: 64 sequences of 1900 .. 6000 keys, 8 heads of 128 at 8 bits, bf16 (545 MB): 102 us, 5.3 TB/s; one of 130001 keys at
// 4 bits (143 MB): 37.5 us, 3.8 TB/s; the join after either 7 us.
template <int DT, int DH, int BITS, int RT>
struct FewCfg {
    static constexpr size_t Q_LDS = (size_t)Wave<DT, DH, BITS, RT>::NP * 16 * RT * QP<DH> * 2;
    static constexpr size_t O_LDS = (size_t)4 * 16 * RT * (DH + 4) * 4;
    static constexpr size_t LDS = Q_LDS > O_LDS ? Q_LDS : O_LDS;
};

template <int DT, int DH, int BITS, int RT, int OCC, bool SCAN>
__global__ __launch_bounds__(256, OCC) void attn_few_kernel(CacheArgs g, const void *__restrict__ yv, int64_t ldy,
                                                          void *__restrict__ av, float *__restrict__ parts,
                                                          Piece *__restrict__ pieces) {
    typedef Wave<DT, DH, BITS, RT> W;
    typedef Lay<DH, BITS> L;
    constexpr int QMID = (1 << (BITS - 1)) - 1, ROWS = 16 * RT;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float rowf[ROWS];
    __shared__ float ml[4][ROWS][2];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int l16 = lane & 15, grp = lane >> 4;
    const int G = g.n_heads / g.n_kv_heads;
    const bool asym = g.k_zero != nullptr;
    const int share = SCAN ? share_of(blockIdx.x, gridDim.x) : blockIdx.x;
    Share<ROWS, SCAN> sh;
    sh.find(g, G, share, gridDim.x, lane);
    if (SCAN && threadIdx.x == 0) pieces[2 * share].flag = pieces[2 * share + 1].flag = 0;

    while (sh.left > 0 && sh.h < g.n_kv_heads) {
        const int s = sh.s, h = sh.h;
        const SeqRows sr = seq_rows(g, s);
        const int n_rows = sr.n * G, row0 = sh.tile * ROWS, nb = tile_blocks<ROWS>(g, sr, G, sh.tile);
        const int b0 = sh.blk, end = (int)min(b0 + sh.left, (int64_t)nb);
        float *part = nullptr;
        if (SCAN && (b0 > 0 || end < nb)) {
            const int slot = 2 * share + (b0 == 0);
            part = parts + (int64_t)slot * ROWS * (DH + 4);
            if (threadIdx.x == 0) pieces[slot] = Piece{s, h, sh.tile, end < nb ? 1 : 2};
        }
        sh.left -= end - b0;
        sh.advance(g, G);
        W w;
        w.limits(g, sr, G, row0, n_rows, l16);
        u32x2 k[2][L::KU], v[L::VU], vz = {0, 0};
        f32x4 ks[2], vs[2];
        int kz[2] = {QMID, QMID};
        // a lane's byte offsets inside a block; its first slot is wave-uniform
        const uint32_t zoff = L::key(0, l16), koff = zoff * L::DHB + L::kbyte(0, grp), voff = L::vrow(0, l16) * 32 + 8 * grp;
        auto load_k = [&](int64_t slot) {
            const uint8_t *kb = g.k + slot * L::DHB, *sb = reinterpret_cast<const uint8_t *>(g.k_scale + slot);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int u = 0; u < L::KU; u += 2) {
                    if constexpr (L::KU >= 2) {            // two units are 16 bytes
                        const u32x4 q = ldu_once<u32x4>(kb, koff + 4 * t * L::DHB + 64 * (u >> 1));
                        k[t][u] = u32x2{q[0], q[1]};
                        k[t][u + 1] = u32x2{q[2], q[3]};
                    } else {
                        k[t][0] = ldu_once<u32x2>(kb, koff + 4 * t * L::DHB);
                    }
                }
                if (asym) kz[t] = ldu_once<uint8_t>(g.k_zero + slot, zoff + 4 * t);
                ks[t] = ldu_once<f32x4>(sb, 32 * grp + 16 * t);
            }
        };
        auto load_v = [&](int64_t slot) {
            const uint8_t *vb = g.v + slot * L::DHB, *sb = reinterpret_cast<const uint8_t *>(g.v_scale + slot);
#pragma unroll
            for (int u = 0; u < L::VU; ++u) v[u] = ldu_once<u32x2>(vb, voff + 512 * u);
#pragma unroll
            for (int t = 0; t < 2; ++t) vs[t] = ldu_once<f32x4>(sb, 32 * grp + 16 * t);
            if (asym) vz = ldu_once<u32x2>(g.v_zero + slot, 8 * grp);
        };
        // blocks wave, wave + 4, ... of the piece, the first one's bytes on their way before the queries are made; a
        // block without a page, and past the end, loads page 0 and is not used
        int b = b0 + wave;
        int64_t slot = b < end ? block_slot(g, s, h, b) : -1;
        load_k(max(slot, (int64_t)0));
        load_v(max(slot, (int64_t)0));
        __builtin_amdgcn_sched_barrier(0);

        _Float16 *ql = reinterpret_cast<_Float16 *>(smem);
        __syncthreads();                                   // LDS of the tile before
        // rows that do not exist keep what LDS holds: a row is one column of every product, and theirs are not stored
#pragma unroll 1
        for (int r = wave; r < ROWS; r += 4) {
            float f = 0.f;
            if (row0 + r < n_rows) f = query_row<DT, DH, W::NP>(g, sr, yv, ldy, h, G, row0 + r, ql, r, ROWS * QP<DH>, lane);
            if (lane == 0) rowf[r] = f;
        }
        __syncthreads();
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            w.fs[rt] = rowf[16 * rt + l16];
#pragma unroll
            for (int p = 0; p < W::NP; ++p)
#pragma unroll
                for (int ks = 0; ks < L::KS; ++ks)
                    w.qf[rt][p][ks] = *reinterpret_cast<const f16x8 *>(ql + p * ROWS * QP<DH> + (16 * rt + l16) * QP<DH> + L::dim(ks, grp));
        }
        w.start();
        if (b < end) {
            for (;;) {
                const bool more = b + 4 < end;
                const int64_t next = more ? block_slot(g, s, h, b + 4) : -1;
                // no page: nothing of the block is seen
                const int key0 = slot >= 0 ? b * 32 + 8 * grp : NOWHERE;
                const bool edge = slot < 0 || b * 32 + 31 > w.lo_lim;
                f32x4 st[RT][2];
                f16x8 pw[RT][W::NP];
                f16x2 zk[2][4];
#pragma unroll
                for (int t = 0; t < 2; ++t) zk[t][0] = zk[t][1] = zk[t][2] = zk[t][3] = both(kz[t]);
                w.scores(st, [&](int t, int step) { return L::kop(k[t], step, grp, zk[t]); });
                w.scale(st, ks);
                w.mask(st, edge, key0);
                __builtin_amdgcn_sched_barrier(0);
                load_k(max(next, (int64_t)0));             // after the last block: page 0, not used
                __builtin_amdgcn_sched_barrier(0);
                float vsc[8];
                w.value_scales(st, vs, edge, key0, vsc);
                w.move(st, vsc);
                const float up = w.up();
#pragma unroll
                for (int i = 0; i < 8; ++i) vsc[i] *= up;
#pragma unroll
                for (int j = 0; j < 4 * RT; ++j) w.weight2(j, st, vsc, pw);
                f16x2 zv[4] = {biased(vz[0], false), biased(vz[0], true), biased(vz[1], false), biased(vz[1], true)};
                if (!asym) zv[0] = zv[1] = zv[2] = zv[3] = both(QMID);
                w.values(pw, [&](int t) { return L::vop(v, t, l16, zv); });
                __builtin_amdgcn_sched_barrier(0);
                if (!more) break;
                load_v(max(next, (int64_t)0));
                __builtin_amdgcn_sched_barrier(0);
                slot = next;
                b += 4;
            }
        }
        w.finish();

        // ---- the four waves' sums, through LDS
        float *ol = reinterpret_cast<float *>(smem);
        __syncthreads();                                   // every wave has its queries
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (grp == 0) {
                ml[wave][16 * rt + l16][0] = w.m[rt];
                ml[wave][16 * rt + l16][1] = w.l[rt];
            }
#pragma unroll
            for (int t = 0; t < L::NT; ++t)
                *reinterpret_cast<f32x4 *>(ol + (wave * ROWS + 16 * rt + l16) * (DH + 4) + 16 * t + 4 * grp) = w.o[rt][t];
        }
        __syncthreads();
        const int live = min(ROWS, n_rows - row0);
        for (int c = threadIdx.x; c < live * (DH / 4); c += 256) {
            const int r = c / (DH / 4), d = c % (DH / 4) * 4;
            float mm = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < 4; ++i) mm = fmaxf(mm, ml[i][r][0]);
            f32x4 sum = f32x4{0.f, 0.f, 0.f, 0.f};
            float ll = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // a wave without a key has m = -inf, l = 0; a NaN row keeps m = -inf and l = NaN
                const float f = ml[i][r][0] == mm ? 1.f : exp2f(ml[i][r][0] - mm);
                const f32x4 x = *reinterpret_cast<const f32x4 *>(ol + (i * ROWS + r) * (DH + 4) + d);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += f * x[e];
                ll += f * ml[i][r][1];
            }
            put_row<DT, DH>(g, sr, h, G, row0, r, d, sum, mm, ll, av, part);
        }
    }
}

// ---------------------------------------------------------------- many rows
// Each wave has 32 rows of its own; the workgroup turns a block of 32 tokens at a time into operands in LDS, which its
// four waves share (waves 0, 1 the two key tiles, 2, 3 half of the values each; an operand is 64 lanes x 16 bytes, written
// and read without conflicts).  Three blocks in a ring, one barrier per block; bytes are asked for two blocks before
// they are turned, page numbers before that.  The scores of the next block are formed beside the weights of this one,
// and the next but one is turned beside this one's second product, so that matrix and vector instructions of one wave overlap.
template <int DT, int DH, int BITS>
struct ManyCfg {
    typedef Lay<DH, BITS> L;
    static constexpr int RT = 2, ROWS = 128;
    static constexpr int KOPS = 2 * L::KS, OPS = KOPS + L::NT;                   // operands of a block
    static constexpr int BLOCK = OPS * 1024 + 256;                               // and its 32 + 32 scales
    static constexpr size_t Q_LDS = (size_t)Wave<DT, DH, BITS, RT>::NP * 4 * 16 * QP<DH> * 2;
    static constexpr size_t LDS = 3 * BLOCK > Q_LDS ? 3 * BLOCK : Q_LDS;
};

template <int DT, int DH, int BITS, bool SCAN>
__global__ __launch_bounds__(256, 2) void attn_many_kernel(CacheArgs g, const void *__restrict__ yv, int64_t ldy,
                                                           void *__restrict__ av, float *__restrict__ parts,
                                                           Piece *__restrict__ pieces) {
    typedef ManyCfg<DT, DH, BITS> S;
    typedef Wave<DT, DH, BITS, S::RT> W;
    typedef Lay<DH, BITS> L;
    constexpr int QMID = (1 << (BITS - 1)) - 1, RT = S::RT;
    constexpr int VH = L::VU < 2 ? 1 : L::VU / 2;          // value units of a wave
    constexpr int RU = VH;                                 // units of a wave
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float rowf[64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int l16 = lane & 15, grp = lane >> 4;
    const int G = g.n_heads / g.n_kv_heads;
    const bool asym = g.k_zero != nullptr;
    const int kind = wave >> 1, mine = wave & 1;           // what this wave turns: keys or values, which half
    // (the symmetric grid has no zero-points: bytes that exist are read in their place, and not used)
    const uint8_t *code_base = kind ? g.v : g.k, *zero_base = !asym ? code_base : kind ? g.v_zero : g.k_zero;
    const uint8_t *scale_base = reinterpret_cast<const uint8_t *>(kind ? g.v_scale : g.k_scale);
    // a lane's byte offsets inside a block
    const uint32_t off = kind ? L::vrow(0, l16) * 32 + 8 * grp + (L::VU < 2 ? 0 : mine * VH * 512)
                              : L::key(mine, l16) * L::DHB + L::kbyte(0, grp);
    const uint32_t zoff = kind ? 8 * grp : L::key(mine, l16) & ~3u, zoff2 = kind ? zoff + 4 : zoff;
    const int zsh = kind ? 0 : 8 * (L::key(mine, l16) & 3);
    static_assert(DH < 64 || L::KU == VH, "keys and values alike");
    const int first = kind ? S::KOPS + (DH < 64 ? 0 : mine * VH) : mine * L::KS, high = kind ? L::NT / 2 : L::KU;
    const int nib = kind ? (l16 >> 3) * 4 : (grp & 1) * 4;
    const int share = SCAN ? share_of(blockIdx.x, gridDim.x) : blockIdx.x;
    Share<S::ROWS, SCAN> sh;
    sh.find(g, G, share, gridDim.x, lane);
    if (SCAN && threadIdx.x == 0) pieces[2 * share].flag = pieces[2 * share + 1].flag = 0;

    while (sh.left > 0 && sh.h < g.n_kv_heads) {
        const int s = sh.s, h = sh.h;
        const SeqRows sr = seq_rows(g, s);
        const int n_rows = sr.n * G, tile0 = sh.tile * S::ROWS, row0 = tile0 + wave * 16 * RT;
        const int nb = tile_blocks<S::ROWS>(g, sr, G, sh.tile), b0 = sh.blk, end = (int)min(b0 + sh.left, (int64_t)nb);
        float *part = nullptr;
        if (SCAN && (b0 > 0 || end < nb)) {
            const int slot = 2 * share + (b0 == 0);
            part = parts + (int64_t)slot * S::ROWS * (DH + 4);
            if (threadIdx.x == 0) pieces[slot] = Piece{s, h, sh.tile, end < nb ? 1 : 2};
        }
        sh.left -= end - b0;
        sh.advance(g, G);

        // ---- this wave's share of a block's bytes
        struct Bytes {
            u32x2 u[RU], z;
            float sc;
        } raw;
        auto page_at = [&](int b) {
            const int p = page_of(g, s, min(b, end - 1) * 32);
            return b < end ? p : -1;
        };
        auto load = [&](Bytes &r, int b, int page) {       // (no page, or past the end: page 0, not used)
            const int64_t at = (((int64_t)max(page, 0) * g.n_kv_heads + h) << g.page_shift) +
                               ((b * 32) & ((1 << g.page_shift) - 1));
            const uint8_t *codes = code_base + at * L::DHB;
#pragma unroll
            for (int u = 0; u < RU; ++u) {
                const uint32_t ko = L::kbyte(u, 0), vo = 512 * u;
                r.u[u] = ldu<u32x2>(codes, off + (kind ? vo : ko));
            }
            r.z[0] = ldu<uint32_t>(zero_base + at, zoff);
            r.z[1] = ldu<uint32_t>(zero_base + at, zoff2);
            r.sc = ldu<float>(scale_base + 4 * at, 4 * (lane & 31));
        };
        // the operands of this wave's bytes, keys and values alike (no branch: the loop's instructions are one
        // block to schedule): unit u is operand first + u, at 4 bits its high halves operand first + u + high
        f16x2 z[4];
        auto turn_zero = [&](const Bytes &r) {
            const uint32_t kz = ((r.z[0] >> zsh) & 255u) * 0x01010101u, mid = QMID * 0x01010101u;
            const uint32_t z0 = !asym ? mid : kind ? r.z[0] : kz, z1 = !asym ? mid : kind ? r.z[1] : kz;
            z[0] = biased(z0, false);
            z[1] = biased(z0, true);
            z[2] = biased(z1, false);
            z[3] = biased(z1, true);
        };
        auto turn_unit = [&](const Bytes &r, int u, unsigned char *blk) {
            unsigned char *dst = blk + first * 1024 + lane * 16;
            const uint32_t w0 = r.u[u][0], w1 = r.u[u][1];
            if constexpr (BITS == 8) {
                *reinterpret_cast<f16x8 *>(dst + u * 1024) = codes8(w0, w1, z);
            } else if constexpr (DH < 64) {
                *reinterpret_cast<f16x8 *>(dst) = codes8((w0 >> nib) & 0x0F0F0F0Fu, (w1 >> nib) & 0x0F0F0F0Fu, z);
            } else {
                *reinterpret_cast<f16x8 *>(dst + u * 1024) = codes8(w0 & 0x0F0F0F0Fu, w1 & 0x0F0F0F0Fu, z);
                *reinterpret_cast<f16x8 *>(dst + (u + high) * 1024) =
                    codes8((w0 >> 4) & 0x0F0F0F0Fu, (w1 >> 4) & 0x0F0F0F0Fu, z);
            }
        };
        auto turn_scales = [&](const Bytes &r, unsigned char *blk) {             // (by both waves of a kind: the same)
            *reinterpret_cast<float *>(blk + S::OPS * 1024 + kind * 128 + (lane & 31) * 4) = r.sc;
        };
        auto turn_block = [&](const Bytes &r, unsigned char *blk) {
            turn_zero(r);
#pragma unroll
            for (int u = 0; u < RU; ++u) turn_unit(r, u, blk);
            turn_scales(r, blk);
        };
        // pages of blocks b .. b + 5 as b advances (scalar loads); bytes of b + 2 and b + 3 in registers
        int pg[5];
#pragma unroll
        for (int i = 0; i < 5; ++i) pg[i] = page_at(b0 + i);
        load(raw, b0, pg[0]);

        // ---- queries
        W w;
        _Float16 *ql = reinterpret_cast<_Float16 *>(smem) + wave * 16 * QP<DH>;
        constexpr int QSTRIDE = 4 * 16 * QP<DH>;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            __syncthreads();                               // LDS of the tile before, and of the rows before
            query_rows16<DT, DH, W::NP>(g, sr, yv, ldy, h, G, row0 + 16 * rt, n_rows, ql, QSTRIDE, rowf + wave * 16, lane);
            __syncthreads();
            w.fs[rt] = rowf[wave * 16 + l16];
#pragma unroll
            for (int p = 0; p < W::NP; ++p)
#pragma unroll
                for (int ks = 0; ks < L::KS; ++ks)
                    w.qf[rt][p][ks] = *reinterpret_cast<const f16x8 *>(ql + p * QSTRIDE + l16 * QP<DH> + L::dim(ks, grp));
        }
        __syncthreads();                                   // the ring lies over the queries
        w.limits(g, sr, G, row0, n_rows, l16);
        w.start();

        int slot = 0;                                      // byte offset of block b in the ring
        auto next = [&](int at) { return at == 2 * S::BLOCK ? 0 : at + S::BLOCK; };
        turn_block(raw, smem);
        load(raw, b0 + 1, pg[1]);
        turn_block(raw, smem + S::BLOCK);
        load(raw, b0 + 2, pg[2]);
        __syncthreads();

        // block b's scores (scaled and masked) and value scales, as the loop's body for b wants them
        constexpr int NQ = 2 * L::KS, PF = 2;              // operands read ahead (3 or 4: no faster)
        f32x4 st[RT][2];
        float vs[8];
        auto operand = [&](const unsigned char *blk, int i) { return *reinterpret_cast<const f16x8 *>(blk + i * 1024 + lane * 16); };
        auto product = [&](f32x4 (&to)[RT][2], int i, f16x8 k) {       // key operand i
            const int t = i / L::KS, ks = i % L::KS;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int p = 0; p < W::NP; ++p)
                    to[rt][t] = mma16(k, w.qf[rt][p][ks], ks == 0 && p == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : to[rt][t]);
        };
        auto mask = [&](f32x4 (&to)[RT][2], int b, int page) {
            const bool edge = page < 0 || b * 32 + 31 > w.lo_lim;
            const int key0 = page < 0 ? NOWHERE : b * 32 + 8 * grp;
            w.mask(to, edge, key0);
            const f32x4 v[2] = {f32x4{vs[0], vs[1], vs[2], vs[3]}, f32x4{vs[4], vs[5], vs[6], vs[7]}};
            w.value_scales(to, v, edge, key0, vs);
        };
        auto scales = [&](const unsigned char *blk, int i) {           // two times 16 bytes of key, then of value scales
            return *reinterpret_cast<const f32x4 *>(blk + S::OPS * 1024 + (i >> 1) * 128 + 32 * grp + 16 * (i & 1));
        };
        {
#pragma unroll
            for (int i = 0; i < NQ; ++i) product(st, i, operand(smem, i));
            const f32x4 ks[2] = {scales(smem, 0), scales(smem, 1)};
            w.scale(st, ks);
#pragma unroll
            for (int i = 0; i < 8; ++i) vs[i] = scales(smem, 2 + (i >> 2))[i & 3];
            mask(st, b0, pg[0]);
        }
        for (int b = b0; b < end; ++b) {
            const unsigned char *cur = smem + slot, *nxt = smem + next(slot);
            unsigned char *fill = smem + next(next(slot));
            f16x8 op[NQ > L::NT ? NQ : L::NT];
#pragma unroll
            for (int i = 0; i < PF; ++i) op[i] = operand(nxt, i);
            w.move(st, vs);
            const float up = w.up();
#pragma unroll
            for (int i = 0; i < 8; ++i) vs[i] *= up;
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);                 // before the other workgroup's waves, which wait for theirs
            // the next block's scores (past the end: of what the ring holds, not used) beside this block's weights
            f32x4 sn[RT][2];
            f16x8 pw[RT][W::NP], vo[L::NT];
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                if (i + PF < NQ) op[i + PF] = operand(nxt, i + PF);
                else if (i + PF - NQ < L::NT) vo[i + PF - NQ] = operand(cur, S::KOPS + i + PF - NQ);
                product(sn, i, op[i]);
#pragma unroll
                for (int j = i * 4 * RT / NQ; j < (i + 1) * 4 * RT / NQ; ++j) w.weight2(j, st, vs, pw);
                __builtin_amdgcn_sched_barrier(0);
            }
            // this block's second product beside the turning of the next but one and the next one's scales
            f32x4 sc4[4];
            turn_zero(raw);
#pragma unroll
            for (int t = 0; t < L::NT; ++t) {
                if (t + PF < L::NT) vo[t + PF] = operand(cur, S::KOPS + t + PF);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int p = 0; p < W::NP; ++p) w.o[rt][t] = mma16(vo[t], pw[rt][p], w.o[rt][t]);
#pragma unroll
                for (int u = t * RU / L::NT; u < (t + 1) * RU / L::NT; ++u) turn_unit(raw, u, fill);
                if (t == 0)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc4[i] = scales(nxt, i);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
            const int ahead = page_at(b + 5);              // (here: no wait for LDS before the barrier waits for it too)
            turn_scales(raw, fill);
            load(raw, b + 3, pg[3]);
            const f32x4 ksn[2] = {sc4[0], sc4[1]};
            w.scale(sn, ksn);
#pragma unroll
            for (int i = 0; i < 8; ++i) vs[i] = sc4[2 + (i >> 2)][i & 3];
            mask(sn, b + 1, pg[1]);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int t = 0; t < 2; ++t) st[rt][t] = sn[rt][t];
#pragma unroll
            for (int i = 0; i < 4; ++i) pg[i] = pg[i + 1];
            pg[4] = ahead;
            slot = next(slot);
            __syncthreads();
        }
        w.finish();
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int row = row0 + 16 * rt + l16;
            if (row < n_rows)
#pragma unroll
                for (int t = 0; t < L::NT; ++t)
                    put_row<DT, DH>(g, sr, h, G, tile0, row - tile0, 16 * t + 4 * grp, w.o[rt][t], w.m[rt], w.l[rt], av, part);
        }
    }
}

// The pieces of the tile that begins in share blockIdx.x and ends in a later one: a wave per row for few pieces, else a
// workgroup, so that a row's loads are in flight together.
constexpr int CUS = 256;
constexpr int MOST_SHARES = 3 * CUS;
template <int DT, int DH, int ROWS>
__global__ __launch_bounds__(256) void attn_join_kernel(CacheArgs g, const float *__restrict__ parts,
                                                        const Piece *__restrict__ pieces, int n_shares, void *__restrict__ av) {
    constexpr int LPR = DH / 4, PITCH = DH + 4;            // lanes of a row's elements
    __shared__ int last_share;
    __shared__ float fac[MOST_SHARES], red[4][2];
    __shared__ f32x4 sum[4][LPR];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int w = blockIdx.x;
    const Piece p = pieces[2 * w + 1];
    if (p.flag != 1) return;
    if (tid == 0) last_share = n_shares;
    __syncthreads();
    for (int i = w + 1 + tid; i < n_shares; i += 256)      // the first end behind it is its own
        if (pieces[2 * i].flag == 2) {
            atomicMin(&last_share, i);
            break;
        }
    __syncthreads();
    const int count = last_share - w + 1;                  // pieces: slot 2 w + 1, then 2 (w + 1), 2 (w + 2), ...
    if (last_share == n_shares) return;
    const SeqRows sr = seq_rows(g, p.s);
    const int G = g.n_heads / g.n_kv_heads, row0 = p.tile * ROWS, live = min(ROWS, sr.n * G - row0);
    auto piece = [&](int i, int r) { return parts + ((int64_t)(i ? 2 * (w + i) : 2 * w + 1) * ROWS + r) * PITCH; };
    if (count <= 8) {                                      // LPR lanes per row, every row's loads in flight at once
        constexpr int RPW = 64 / LPR, STEP = 2;
        const int d = lane % LPR * 4, step = 4 * RPW * gridDim.y;
        for (int r0 = (blockIdx.y * 4 + wave) * RPW + lane / LPR; r0 < live; r0 += STEP * step) {
#pragma unroll
            for (int u = 0; u < STEP; ++u) {
                const int r = r0 + u * step, rr = min(r, live - 1);
                float m = -__builtin_inff(), l = 0.f;
                f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
                for (int i = 0; i < count; ++i) {          // the reference moves with the larger m
                    const float *q = piece(i, rr);
                    const float mi = q[DH], li = q[DH + 1];
                    const f32x4 x = *reinterpret_cast<const f32x4 *>(q + d);
                    const float mn = fmaxf(m, mi), a = m == mn ? 1.f : exp2f(m - mn), b = mi == mn ? 1.f : exp2f(mi - mn);
                    m = mn;
                    l = a * l + b * li;
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = a * v[k] + b * x[k];
                }
                if (r < live) put_row<DT, DH>(g, sr, p.h, G, row0, r, d, v, m, l, av, nullptr);
            }
        }
        return;
    }
    constexpr int SG = 256 / LPR;
    const int d = tid % LPR * 4, sg = tid / LPR;
    for (int r = blockIdx.y; r < live; r += gridDim.y) {
        float mi[MOST_SHARES / 256], li[MOST_SHARES / 256], m = -__builtin_inff(), l = 0.f;
#pragma unroll
        for (int k = 0; k < MOST_SHARES / 256; ++k) {
            const int i = tid + 256 * k;
            mi[k] = i < count ? piece(i, r)[DH] : -__builtin_inff();
            li[k] = i < count ? piece(i, r)[DH + 1] : 0.f;
            m = fmaxf(m, mi[k]);
        }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
        __syncthreads();                                   // the row before is done with red, fac and sum
        if (lane == 0) red[wave][0] = m;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, red[i][0]);
#pragma unroll
        for (int k = 0; k < MOST_SHARES / 256; ++k) {
            const int i = tid + 256 * k;
            const float f = mi[k] == m ? 1.f : exp2f(mi[k] - m);
            if (i < count) fac[i] = f;
            l += f * li[k];
        }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) l += __shfl_xor(l, off, 64);
        if (lane == 0) red[wave][1] = l;
        __syncthreads();
        l = red[0][1] + red[1][1] + red[2][1] + red[3][1];
        f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int i = sg; i < count; i += SG) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(piece(i, r) + d);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += fac[i] * x[k];
        }
#pragma unroll
        for (int off = 32; off >= LPR; off >>= 1)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += __shfl_xor(v[k], off, 64);
        if (lane < LPR) sum[wave][lane] = v;
        __syncthreads();
        if (tid < LPR) {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = (sum[0][tid][k] + sum[1][tid][k]) + (sum[2][tid][k] + sum[3][tid][k]);
            put_row<DT, DH>(g, sr, p.h, G, row0, r, d, v, m, l, av, nullptr);
        }
    }
}

// The kernel and its shares, from the sizes that the host knows.
struct Plan {
    bool few, scan;                     // scan: equal shares of the whole batch, whose pieces are joined
    bool many_pieces;                   // tiles of more than 8 shares are expected
    int rt, rows;                       // few: 16-row tiles of a wave; rows of a tile
    int groups;                         // workgroups = shares
};
Plan plan_of(int dtype, const CacheArgs &g) {
    Plan p;
    const int G = g.n_heads / g.n_kv_heads;
    const int64_t rows = (int64_t)std::max(g.max_new, 1) * G, blocks = ((int64_t)g.cap + 31) / 32;
    // (33 .. 64 rows as two few tiles: fp16 50 instead of 59 us at 8 x 4000 tokens, but bf16 213 instead of 192 at 64 x 4000
    // and 31 instead of 23 at 8 x 400)
    p.few = rows <= 32;
    p.rt = rows <= 16 ? 1 : 2;
    p.rows = p.few ? 16 * p.rt : 128;
    const int64_t pairs = (int64_t)g.n_seq * g.n_kv_heads, tiles = (rows + p.rows - 1) / p.rows;
    // Equal shares, but not where a (sequence, head) is short, nor where there are too many sequences to scan.  A head's
    // blocks of all sequences fit 32 bits (the tiles of all rows, and a ragged one per sequence).
    p.scan = tiles * blocks >= (p.few ? WHOLE_FEW : WHOLE_MANY) && g.n_seq <= SCAN_SEQS &&
             ((int64_t)g.M * G / p.rows + g.n_seq) * blocks < INT32_MAX;
    p.many_pieces = false;
    p.groups = (int)pairs;
    if (!p.scan) return p;
    // one round of the workgroups that the CUs hold at once; fewer where the shares would be short (two rounds: one
    // sequence of 130000 tokens 53 us instead of 43)
    const int64_t slots = (int64_t)CUS * (p.few && p.rt == 1 && dtype == BF16 ? 3 : 2);
    p.groups = (int)std::min(slots, std::max<int64_t>(1, pairs * tiles * blocks / SHARE));
    if (p.groups > 8) p.groups &= ~7;
    p.many_pieces = p.groups > 8 * pairs * tiles;
    return p;
}

template <int DT, int DH, int ROWS, typename K>
hipError_t run_attn(K kernel, size_t lds, const CacheArgs &g, const Plan &p, const void *y, int64_t ldy, void *a, void *ws, hipStream_t st) {
    hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    Piece *pieces = static_cast<Piece *>(ws);
    float *parts = reinterpret_cast<float *>(pieces + 2 * p.groups);
    kernel<<<dim3(p.groups), 256, lds, st>>>(g, y, ldy, a, parts, pieces);
    e = hipGetLastError();
    if (e != hipSuccess || !p.scan || p.groups == 1) return e;
    // the rows that the host expects (others in turn): one workgroup each where a tile has many pieces, else one for
    // what its lanes take at once
    const int rows = (int)std::min<int64_t>(ROWS, (int64_t)std::max(g.max_new, 1) * (g.n_heads / g.n_kv_heads));
    const int at_once = p.many_pieces ? 1 : 4 * (64 / (DH / 4)) * 2;
    attn_join_kernel<DT, DH, ROWS><<<dim3(p.groups - 1, (rows + at_once - 1) / at_once), 256, 0, st>>>(g, parts, pieces, p.groups, a);
    return hipGetLastError();
}

template <int DT, int DH, int BITS>
hipError_t run_plan(const CacheArgs &g, const void *y, int64_t ldy, void *a, void *ws, hipStream_t st) {
    const Plan p = plan_of(DT, g);
    auto run = [&](auto scan) -> hipError_t {
        constexpr bool SCAN = decltype(scan)::value;
        constexpr int OCC1 = DT == BF16 ? 3 : 2, OCC2 = 2;
        if (!p.few)
            return run_attn<DT, DH, 128>(attn_many_kernel<DT, DH, BITS, SCAN>, ManyCfg<DT, DH, BITS>::LDS, g, p, y, ldy, a, ws, st);
        return p.rt == 1 ? run_attn<DT, DH, 16>(attn_few_kernel<DT, DH, BITS, 1, OCC1, SCAN>, FewCfg<DT, DH, BITS, 1>::LDS, g, p, y, ldy, a, ws, st)
                         : run_attn<DT, DH, 32>(attn_few_kernel<DT, DH, BITS, 2, OCC2, SCAN>, FewCfg<DT, DH, BITS, 2>::LDS, g, p, y, ldy, a, ws, st);
    };
    return p.scan ? run(std::true_type()) : run(std::false_type());
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

size_t attn_cache_ws_bytes(int dtype, const CacheArgs &g) {
    const Plan p = plan_of(dtype, g);
    return p.scan ? (size_t)2 * p.groups * (sizeof(Piece) + (size_t)p.rows * (g.head_dim + 4) * sizeof(float)) : 0;
}

hipError_t launch_attn_cache(int dtype, const CacheArgs &g, const void *y, int64_t ldy, void *a, void *ws, hipStream_t st) {
    switch (dtype) {
    case F32: return run_dh<F32>(g, y, ldy, a, ws, st);
    case F16: return run_dh<F16>(g, y, ldy, a, ws, st);
    default: return run_dh<BF16>(g, y, ldy, a, ws, st);
    }
}

}  // namespace jab
