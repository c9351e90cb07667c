// cache.hip -- keys and values quantized into the paged cache, and read back.
//
// Per (token, head) one grid of eq. quant over the head's dh elements, every step correctly rounded in fp32:
//   asymmetric: lo = min(0, min x), hi = max(0, max x), s = (hi - lo) / (2^b - 1), z = clip(RNE(-lo / s), 0, 2^b - 1),
//               code = clip(RNE(x / s) + z, 0, 2^b - 1), value (code - z) s
//   symmetric:  s = max|x| / q, code = clip(RNE(x / s), -q, q) + q, q = 2^(b-1) - 1, value (code - q) s
// (s = 0 counts as 1; a head with an infinite or NaN element, or whose range overflows, gets s = NaN).  Keys
// are first turned by the rotary embedding: angle, cosine, sine and turn in fp64, rounded to fp32 once.
//
// Bound by HBM (the projection's columns in, the codes out).  A workgroup takes blocks of 32 positions of one
// sequence and all heads or a group of them: the fp64 cosines and sines of a block are formed once for its heads.  Eight
// lanes per (token, head), each with the pairs (j, j + dh / 2) that the rotation and the 4-bit bytes
// need; values leave through LDS, where a head's tile turns to the cache's token-contiguous order, and the next head's
// elements are on their way under this one's arithmetic.
// A block with few new tokens (a decoding step) goes by (token, head) items instead, all heads at once.
// Measured: 32768 bf16 tokens of 8 heads of 128 (201 MB both ways) are written in 56-64 us, where memory alone needs 40 and
// the arithmetic, about 8 instructions an element, 35, and read back in 36 (5.6 TB/s).
#include <algorithm>

#include "device_common.h"
#include "cache.h"

namespace jab {
namespace {

constexpr int FEW = 4;                  // new tokens of a block that go without the LDS tile
constexpr int PITCH = 36;               // bytes between the tile's rows of 32 tokens in LDS (words 9 d + t / 4: few conflicts)

// C elements
template <typename E, int C>
__device__ inline void load_c(const E *p, E *e) {
    constexpr int B = C * (int)sizeof(E);
    if constexpr (B % 16 == 0) {
#pragma unroll
        for (int i = 0; i < B / 16; ++i) reinterpret_cast<u32x4 *>(e)[i] = reinterpret_cast<const u32x4 *>(p)[i];
    } else if constexpr (B == 8) {
        *reinterpret_cast<uint2 *>(e) = *reinterpret_cast<const uint2 *>(p);
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) e[i] = p[i];
    }
}
template <int DT, int C>
__device__ inline void store_c(typename Mma<DT>::elem *p, const float *v) {
    typedef typename Mma<DT>::elem elem;
    elem e[C];
    constexpr int B = C * (int)sizeof(elem);
#pragma unroll
    for (int i = 0; i < C; ++i) e[i] = from_f32<DT>(v[i]);
    if constexpr (B % 16 == 0) {
#pragma unroll
        for (int i = 0; i < B / 16; ++i) reinterpret_cast<u32x4 *>(p)[i] = reinterpret_cast<const u32x4 *>(e)[i];
    } else if constexpr (B == 8) {
        *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<const uint2 *>(e);
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) p[i] = e[i];
    }
}
template <int C>
__device__ inline void store_bytes(uint8_t *p, const uint8_t *b) {
    if constexpr (C == 8) {
        uint2 w;
        __builtin_memcpy(&w, b, 8);
        *reinterpret_cast<uint2 *>(p) = w;
    } else if constexpr (C == 4) {
        uint32_t w;
        __builtin_memcpy(&w, b, 4);
        *reinterpret_cast<uint32_t *>(p) = w;
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) p[i] = b[i];
    }
}
template <int C>
__device__ inline void load_bytes(const uint8_t *p, uint8_t *b) {
    if constexpr (C == 8) {
        const uint2 w = *reinterpret_cast<const uint2 *>(p);
        __builtin_memcpy(b, &w, 8);
    } else if constexpr (C == 4) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(p);
        __builtin_memcpy(b, &w, 4);
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) b[i] = p[i];
    }
}

// f over the eight consecutive lanes of a (token, head): every lane gets the whole.
template <typename F>
__device__ inline float over8(float v, F &&f) {
    auto at = [](float x, auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    v = f(v, at(v, std::integral_constant<int, 0xB1>{}));  // neighbours (quad 1 0 3 2)
    v = f(v, at(v, std::integral_constant<int, 0x4E>{}));  // pairs (quad 2 3 0 1)
    return f(v, at(v, std::integral_constant<int, 0x141>{}));   // quads (eight mirrored)
}
// One word of each of four tokens (lanes eight apart), its bytes four elements: the lane of token i gets the
// four tokens' bytes i.  Two steps of a 4 x 4 transposition, lanes 8 and 16 apart.
__device__ inline uint32_t quad_bytes(uint32_t w) {
    const bool b0 = threadIdx.x & 8, b1 = threadIdx.x & 16;
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0x128, 0xF, 0xF, true);     // 8 lanes on
    w = __builtin_amdgcn_perm(o, w, b0 ? 0x03070105u : 0x06020400u);   // bytes of o are 4 .. 7
    uint32_t lo = w, hi = w;                               // words of the even and of the odd rows of 16 lanes
    asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1" : "+v"(lo), "+v"(hi));
    return __builtin_amdgcn_perm(hi, lo, b1 ? 0x07060302u : 0x05040100u);
}

// Codes of the 2 C elements that this lane holds of a head (eight consecutive lanes hold the head), four to a
// word in order, its scale and zero-point.
// Quotients x / s are rounded to fp32 as a division rounds them, without dividing: in fp64, x times the rounded 1 / s is
// within 2^-52 of x / s, and a quotient of two fp32 numbers is nearer than 2^-25 of its last place to no midpoint of
// two fp32 numbers, so both round alike; the same holds of a division by the constants.  (32 divisions of
// a lane were half of the kernel's instructions.)
template <int BITS, int C>
__device__ inline void encode(const float (&x)[2 * C], bool sym, uint32_t (&code)[(2 * C + 3) / 4], float &s, uint8_t &z) {
    float lo = 0.f, hi = 0.f, bad = 0.f;                   // bad: NaN with an infinite or NaN element
#pragma unroll
    for (int i = 0; i < 2 * C; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        bad = __builtin_fmaf(x[i], 0.f, bad);
    }
    lo = over8(lo, [](float a, float b) { return fminf(a, b); });
    hi = over8(hi, [](float a, float b) { return fmaxf(a, b); });
    bad = over8(bad, [](float a, float b) { return a + b; });
    constexpr float top = (float)((1 << BITS) - 1), q = (float)((1 << (BITS - 1)) - 1);
    float zf = q, most = 2.f * q;
    s = (float)(sym ? (double)fmaxf(-lo, hi) * (1.0 / q) : (double)(hi - lo) * (1.0 / top));
    if (s == 0.f) s = 1.f;
    const double r = 1.0 / (double)s;
    if (!sym) {
        zf = fminf(fmaxf(rintf((float)(-(double)lo * r)), 0.f), top);
        most = top;
    }
    if (!(bad == 0.f && s < __builtin_inff())) {
        s = __builtin_nanf("");
        zf = most = 0.f;                                   // and all codes 0: the middle of (0, 0, anything), NaN too
    }
    z = (uint8_t)(int)zf;
#pragma unroll
    for (int w = 0; w < (2 * C + 3) / 4; ++w) code[w] = 0;
#pragma unroll
    for (int i = 0; i < 2 * C; ++i) {
        const float v = __builtin_amdgcn_fmed3f(rintf((float)((double)x[i] * r)) + zf, 0.f, most);
        code[i >> 2] = __builtin_amdgcn_cvt_pk_u8_f32(v, i & 3, code[i >> 2]);
    }
}

// The blocks of 32 positions that hold new tokens of a sequence, dealt out over the workgroups, gridDim.y groups of heads:
// f(sequence, its rows, block, first and one past the last new token inside the block, first and one past the last head)
template <typename F>
__device__ inline void for_blocks(const CacheArgs &g, int nb, F &&f) {
    const uint32_t hg = gridDim.y, grp = blockIdx.y;
    const int h0 = (int)(g.n_kv_heads * grp / hg), h1 = (int)(g.n_kv_heads * (grp + 1) / hg);
    for (int64_t it = blockIdx.x; it < (int64_t)g.n_seq * nb; it += gridDim.x) {
        const int s = it >> 32 ? (int)(it / nb) : (int)((uint32_t)it / (uint32_t)nb);
        const SeqRows r = seq_rows(g, s);
        const int end = (int)min((int64_t)r.past + r.n, (int64_t)g.cap);
        for (int64_t at = (r.past >> 5) + (it - (int64_t)s * nb); at * 32 < end; at += nb) {        // (a step may pass 32 bits of positions)
            const int blk = (int)at;
            const int t0 = max(r.past - blk * 32, 0), t1 = min(end - blk * 32, 32);
            if (t0 < t1) f(s, r, blk, t0, t1, h0, h1);
        }
    }
}

template <int DT, int DH, int BITS>
__global__ __launch_bounds__(256, 4) void cache_write_kernel(CacheArgs g, const void *__restrict__ yv, int64_t ldy, int nb) {
    typedef typename Mma<DT>::elem elem;
    constexpr int HALF = DH / 2, C = DH / 16, DHB = DH * BITS / 8;
    __shared__ double2 tab[32 * HALF];                 // (cos, sin) of the block's positions, pair j of a token at mix(j):
    auto mix = [](int j) { return j ^ ((j >> 3) & 7); };    // the eight lanes of a head read distinct banks
    __shared__ __align__(16) uint8_t tile[DHB * PITCH];
    const int tid = threadIdx.x, e = tid & 7, slot32 = tid >> 3;
    const bool rope = g.freq[0] != 0.0, sym = g.k_zero == nullptr;
    for_blocks(g, nb, [&](int s, const SeqRows &r, int blk, int t0, int t1, int h0, int h1) {
        const int page = page_of(g, s, blk * 32);
        if (page < 0) return;
        const int nt = t1 - t0, at0 = (blk * 32) & ((1 << g.page_shift) - 1);
        if (rope) {
            __syncthreads();
            if (nt <= FEW) {
                for (int i = tid; i < nt * HALF; i += 256) {
                    double sn, cs;
                    sincos((double)(blk * 32 + t0 + i / HALF) * g.freq[i % HALF], &sn, &cs);
                    tab[i / HALF * HALF + mix(i % HALF)] = make_double2(cs, sn);
                }
            } else {
                // eight positions in a row from the first one's angle, each the one before turned by one position (in
                // fp64: 2^-53 a step; a sine and cosine are 250 instructions, a turn 6)
                for (int i = tid; i < 4 * HALF; i += 256) {
                    const int j = i % HALF, k0 = i / HALF * 8;
                    double sn, cs, s1, c1;
                    sincos((double)(blk * 32 + t0 + k0) * g.freq[j], &sn, &cs);
                    sincos(g.freq[j], &s1, &c1);
                    for (int k = k0; k < min(k0 + 8, nt); ++k) {
                        tab[k * HALF + mix(j)] = make_double2(cs, sn);
                        const double c = cs * c1 - sn * s1;
                        sn = sn * c1 + cs * s1;
                        cs = c;
                    }
                }
            }
            __syncthreads();
        }
        const elem *rows = static_cast<const elem *>(yv) + (int64_t)(r.row + (blk * 32 - r.past)) * ldy;
        // one (token, head): its elements; then codes, key bytes and scales stored, value codes returned.  Another one's
        // elements are asked for where this one's are used up, so that they are on their way under the arithmetic.
        struct Elems {
            __align__(16) elem k[2 * C], v[2 * C];
        };
        auto key_at = [&](int t, int h) { return rows + (int64_t)t * ldy + (int64_t)(g.n_heads + h) * DH + e * C; };
        auto load_k = [&](Elems &m, int t, int h) {
            const elem *p = key_at(t, h);
            load_c<elem, C>(p, m.k);
            load_c<elem, C>(p + HALF, m.k + C);
        };
        auto load_v = [&](Elems &m, int t, int h) {
            const elem *p = key_at(t, h) + (int64_t)g.n_kv_heads * DH;
            load_c<elem, C>(p, m.v);
            load_c<elem, C>(p + HALF, m.v + C);
        };
        auto item = [&](Elems &m, int t, int h, int next, uint32_t (&vw)[(2 * C + 3) / 4]) {
            float x[2 * C], y[2 * C];
#pragma unroll
            for (int i = 0; i < 2 * C; ++i) x[i] = to_f32<DT>(m.k[i]);
            if (next >= 0) load_k(m, t, next);
            if (rope) {
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    const double2 cs = tab[(t - t0) * HALF + mix(e * C + i)];
                    const double a = x[i], b = x[C + i];
                    x[i] = (float)(a * cs.x - b * cs.y);
                    x[C + i] = (float)(b * cs.x + a * cs.y);
                }
            }
            uint8_t kc[2 * C], kz, vz;
            uint32_t kw[(2 * C + 3) / 4];
            float ks, vs;
            encode<BITS, C>(x, sym, kw, ks, kz);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 2 * C; ++i) y[i] = to_f32<DT>(m.v[i]);
            if (next >= 0) load_v(m, t, next);
            encode<BITS, C>(y, sym, vw, vs, vz);
            __builtin_memcpy(kc, kw, 2 * C);
            const int64_t slot = (((int64_t)page * g.n_kv_heads + h) << g.page_shift) + at0 + t;
            uint8_t *kr = g.k + slot * DHB + e * C;
            if constexpr (BITS == 8) {
                store_bytes<C>(kr, kc);
                store_bytes<C>(kr + HALF, kc + C);
            } else {
                if constexpr (C >= 4) {
#pragma unroll
                    for (int i = 0; i < C / 4; ++i) {
                        kw[i] |= kw[C / 4 + i] << 4;
                        vw[i] |= vw[C / 4 + i] << 4;
                    }
                    __builtin_memcpy(kc, kw, C);
                } else {
                    kc[0] |= kc[1] << 4;
                    vw[0] = (vw[0] | vw[0] >> 4) & 255u;
                }
                store_bytes<C>(kr, kc);
            }
            if (e == 0) g.k_scale[slot] = ks;
            if (e == 1) g.v_scale[slot] = vs;
            if (!sym) {
                if (e == 2) g.k_zero[slot] = kz;
                if (e == 3) g.v_zero[slot] = vz;
            }
        };
        constexpr int NC = BITS == 8 ? 2 * C : C;      // value bytes of a lane, rows e C + i (and HALF + e C + i)
        auto vbase = [&](int h) {
            return g.v + ((((int64_t)page * g.n_kv_heads + h) << g.page_shift) + at0) * DHB;
        };
        if (nt <= FEW) {
            for (int i0 = 0; i0 < nt * (h1 - h0); i0 += 32) {
                const int i = i0 + slot32;
                if (i >= nt * (h1 - h0)) break;     // eight lanes of an item leave together
                const int t = t0 + i % nt, h = h0 + i / nt;
                uint32_t vw[(2 * C + 3) / 4];
                Elems m;
                load_k(m, t, h);
                load_v(m, t, h);
                item(m, t, h, -1, vw);
                uint8_t *vb = vbase(h);
#pragma unroll
                for (int k = 0; k < NC; ++k)
                    vb[(e * C + (k < C ? k : HALF + k - C)) * 32 + t] = (uint8_t)(vw[k >> 2] >> (8 * (k & 3)));
            }
            return;
        }
        // the lanes of four tokens exchange their bytes, so that a word of the tile is four tokens of one element (tokens
        // that are not new leave what is not stored)
        const int t = slot32;
        const bool mine = t >= t0 && t < t1;
        Elems m;
        if (mine) {
            load_k(m, t, h0);
            load_v(m, t, h0);
        }
        for (int h = h0; h < h1; ++h) {
            uint32_t vw[(2 * C + 3) / 4] = {};
            if (mine) item(m, t, h, h + 1 < h1 ? h + 1 : -1, vw);
            if (h > h0) __syncthreads();                      // the tile is read
#pragma unroll
            for (int w = 0; w < (NC + 3) / 4; ++w) {
                const uint32_t q = quad_bytes(vw[w]);
                const int k = 4 * w + (t & 3);             // this lane's element of the word
                if (NC % 4 == 0 || k < NC)
                    *reinterpret_cast<uint32_t *>(tile + (e * C + (k < C ? k : HALF + k - C)) * PITCH + (t & ~3)) = q;
            }
            __syncthreads();
            uint8_t *vb = vbase(h);
            for (int w = tid; w < DHB * 8; w += 256) { // words of four tokens; an edge word goes by bytes
                const int d = w >> 3, tw = (w & 7) * 4;
                const uint8_t *src = tile + d * PITCH + tw;
                if (tw >= t0 && tw + 4 <= t1) {
                    *reinterpret_cast<uint32_t *>(vb + d * 32 + tw) = *reinterpret_cast<const uint32_t *>(src);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (tw + k >= t0 && tw + k < t1) vb[d * 32 + tw + k] = src[k];
                }
            }
        }
        __syncthreads();                                   // the tiles before the next block's
    });
}

template <int DT, int DH, int BITS>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheArgs g, void *__restrict__ kv, void *__restrict__ vv, int nb) {
    typedef typename Mma<DT>::elem elem;
    constexpr int HALF = DH / 2, C = DH / 16, DHB = DH * BITS / 8;
    constexpr int NC = BITS == 8 ? 2 * C : C;
    __shared__ __align__(16) uint8_t tile[DHB * PITCH];
    const int tid = threadIdx.x, e = tid & 7;
    const int64_t ld = (int64_t)g.n_kv_heads * DH;
    constexpr int QMID = (1 << (BITS - 1)) - 1;
    for_blocks(g, nb, [&](int s, const SeqRows &r, int blk, int t0, int t1, int h0, int h1) {
        const int page = page_of(g, s, blk * 32);
        const int nt = t1 - t0, at0 = (blk * 32) & ((1 << g.page_shift) - 1);
        const int64_t row0 = r.row + (blk * 32 - r.past);
        auto value = [&](const uint8_t *c, float sc, int z, float *x) {   // C bytes (low, high) or 2 C codes
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const int a = BITS == 8 ? c[i] : c[i] & 15, b = BITS == 8 ? c[C + i] : c[i] >> 4;
                x[i] = (float)(a - z) * sc;
                x[C + i] = (float)(b - z) * sc;
                // the product is rounded to fp32 before the dtype (the compiler would fuse it with the
                // conversion to fp16, which rounds once)
                asm("" : "+v"(x[i]), "+v"(x[C + i]));
            }
        };
        // the key row, and the value row whose bytes get() fetches
        auto item = [&](int t, int h, auto get) {
            elem *ko = static_cast<elem *>(kv) + (row0 + t) * ld + (int64_t)h * DH + e * C;
            elem *vo = static_cast<elem *>(vv) + (row0 + t) * ld + (int64_t)h * DH + e * C;
            float x[2 * C], y[2 * C];
#pragma unroll
            for (int i = 0; i < 2 * C; ++i) x[i] = y[i] = 0.f;
            if (page >= 0) {
                const int64_t slot = (((int64_t)page * g.n_kv_heads + h) << g.page_shift) + at0 + t;
                const uint8_t *kr = g.k + slot * DHB + e * C;
                uint8_t kc[2 * C], vc[2 * C];
                load_bytes<C>(kr, kc);
                if constexpr (BITS == 8) load_bytes<C>(kr + HALF, kc + C);
#pragma unroll
                for (int k = 0; k < NC; ++k) vc[k] = get(e * C + (k < C ? k : HALF + k - C));
                value(kc, g.k_scale[slot], g.k_zero ? g.k_zero[slot] : QMID, x);
                value(vc, g.v_scale[slot], g.v_zero ? g.v_zero[slot] : QMID, y);
            }
            store_c<DT, C>(ko, x);
            store_c<DT, C>(ko + HALF, x + C);
            store_c<DT, C>(vo, y);
            store_c<DT, C>(vo + HALF, y + C);
        };
        auto vbase = [&](int h) {
            return g.v + ((((int64_t)max(page, 0) * g.n_kv_heads + h) << g.page_shift) + at0) * DHB;
        };
        if (nt <= FEW) {
            for (int i0 = 0; i0 < nt * (h1 - h0); i0 += 32) {
                const int i = i0 + (tid >> 3);
                if (i >= nt * (h1 - h0)) break;
                const int t = t0 + i % nt, h = h0 + i / nt;
                const uint8_t *vb = vbase(h);
                item(t, h, [&](int d) { return vb[d * 32 + t]; });
            }
            return;
        }
        const int t = tid >> 3;
        for (int h = h0; h < h1; ++h) {
            const uint8_t *vb = vbase(h);
            for (int c = tid; c < DHB * 2; c += 256) { // whole tiles: chunks of 16 tokens
                const u32x4 q = *reinterpret_cast<const u32x4 *>(vb + c * 16);
                uint32_t *dst = reinterpret_cast<uint32_t *>(tile + (c >> 1) * PITCH + (c & 1) * 16);
#pragma unroll
                for (int i = 0; i < 4; ++i) dst[i] = q[i];
            }
            __syncthreads();
            if (t >= t0 && t < t1) item(t, h, [&](int d) { return tile[d * PITCH + t]; });
            __syncthreads();
        }
    });
}

// blocks of 32 positions that max_new tokens can touch, and the launch's workgroups (at most 2^20 of them: a workgroup
// takes the next blocks in turn)
int blocks_per_seq(const CacheArgs &g) { return (int)(((int64_t)g.max_new + 62) / 32); }
// Groups of heads for about 1024 workgroups, four per CU: 8 sequences of 5788 tokens, 12 heads of 64, fp16 at 4 bits: 12.8
// and 9.1 us to write and read back, 19.4 and 15.0 with all heads to a workgroup, 14.2 and 10.2 with 4096.  Not for few
// tokens, whose heads a workgroup takes at once (48 x 8 heads of 128: 6.4 us in one group, 7.9 in eight).
dim3 grid_of(const CacheArgs &g) {
    const int64_t n = (int64_t)g.n_seq * blocks_per_seq(g);
    const int64_t hg = g.max_new <= FEW ? 1 : std::max<int64_t>(1, std::min<int64_t>(g.n_kv_heads, 1024 / n));
    return dim3((unsigned)(n < (1 << 20) ? n : (1 << 20)), (unsigned)hg);
}

template <int DT, int DH, int BITS>
hipError_t run_write(const CacheArgs &g, const void *y, int64_t ldy, hipStream_t st) {
    cache_write_kernel<DT, DH, BITS><<<grid_of(g), 256, 0, st>>>(g, y, ldy, blocks_per_seq(g));
    return hipGetLastError();
}
template <int DT, int DH, int BITS>
hipError_t run_read(const CacheArgs &g, void *k, void *v, hipStream_t st) {
    cache_read_kernel<DT, DH, BITS><<<grid_of(g), 256, 0, st>>>(g, k, v, blocks_per_seq(g));
    return hipGetLastError();
}

template <int DT, typename F>
hipError_t by_shape(const CacheArgs &g, F &&f) {
    auto bits = [&](auto dh) -> hipError_t {
        return g.bits == 8 ? f(dh, std::integral_constant<int, 8>()) : f(dh, std::integral_constant<int, 4>());
    };
    switch (g.head_dim) {
    case 16: return bits(std::integral_constant<int, 16>());
    case 64: return bits(std::integral_constant<int, 64>());
    default: return bits(std::integral_constant<int, 128>());
    }
}
template <typename F>
hipError_t by_dtype(int dtype, F &&f) {
    switch (dtype) {
    case F32: return f(std::integral_constant<int, F32>());
    case F16: return f(std::integral_constant<int, F16>());
    default: return f(std::integral_constant<int, BF16>());
    }
}
}  // namespace

hipError_t launch_cache_write(int dtype, const CacheArgs &g, const void *y, int64_t ldy, hipStream_t st) {
    return by_dtype(dtype, [&](auto dt) -> hipError_t {
        constexpr int DT = decltype(dt)::value;
        return by_shape<DT>(g, [&](auto dh, auto b) { return run_write<DT, decltype(dh)::value, decltype(b)::value>(g, y, ldy, st); });
    });
}

hipError_t launch_cache_read(int dtype, const CacheArgs &g, void *k_out, void *v_out, hipStream_t st) {
    return by_dtype(dtype, [&](auto dt) -> hipError_t {
        constexpr int DT = decltype(dt)::value;
        return by_shape<DT>(g, [&](auto dh, auto b) { return run_read<DT, decltype(dh)::value, decltype(b)::value>(g, k_out, v_out, st); });
    });
}

}  // namespace jab
