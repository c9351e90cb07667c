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
// sequence, all heads: the fp64 cosines and sines of a block are formed once for its heads.  Eight
// lanes per (token, head), each with the pairs (j, j + dh / 2) that the rotation and the 4-bit bytes
// need; values leave through LDS, where a head's tile turns to the cache's token-contiguous order.
// A block with few new tokens (a decoding step) goes by (token, head) items instead, all heads at once.
#include "device_common.h"
#include "cache.h"

namespace jab {
namespace {

constexpr int FEW = 4;                  // new tokens of a block that go without the LDS tile
constexpr int PITCH = 40;               // bytes between the tile's rows of 32 tokens in LDS

// C elements as fp32
template <int DT, int C>
__device__ inline void load_c(const typename Mma<DT>::elem *p, float *v) {
    typedef typename Mma<DT>::elem elem;
    elem e[C];
    constexpr int B = C * (int)sizeof(elem);
    if constexpr (B % 16 == 0) {
#pragma unroll
        for (int i = 0; i < B / 16; ++i) reinterpret_cast<u32x4 *>(e)[i] = reinterpret_cast<const u32x4 *>(p)[i];
    } else if constexpr (B == 8) {
        *reinterpret_cast<uint2 *>(e) = *reinterpret_cast<const uint2 *>(p);
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) e[i] = p[i];
    }
#pragma unroll
    for (int i = 0; i < C; ++i) v[i] = to_f32<DT>(e[i]);
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

// codes of the 2 C elements that this lane holds of a head (eight consecutive lanes hold the head), its
// scale and zero-point
template <int BITS, int C>
__device__ inline void encode(const float (&x)[2 * C], bool sym, uint8_t (&code)[2 * C], float &s, uint8_t &z) {
    float lo = 0.f, hi = 0.f;
    uint32_t mx = 0;                    // the largest magnitude, infinity and NaN above all others
#pragma unroll
    for (int i = 0; i < 2 * C; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        mx = max(mx, __builtin_bit_cast(uint32_t, x[i]) & 0x7FFFFFFFu);
    }
#pragma unroll
    for (int off = 1; off < 8; off *= 2) {
        lo = fminf(lo, __shfl_xor(lo, off, 64));
        hi = fmaxf(hi, __shfl_xor(hi, off, 64));
        mx = max(mx, (uint32_t)__shfl_xor((int)mx, off, 64));
    }
    constexpr float top = (float)((1 << BITS) - 1), q = (float)((1 << (BITS - 1)) - 1);
    float zf = q, most = 2.f * q;
    if (sym) {
        s = __builtin_bit_cast(float, mx) / q;
        if (s == 0.f) s = 1.f;
    } else {
        s = (hi - lo) / top;
        if (s == 0.f) s = 1.f;
        zf = fminf(fmaxf(rintf(-lo / s), 0.f), top);
        most = top;
    }
    const bool fine = mx < 0x7F800000u && s < __builtin_inff();
    if (!fine) {
        s = __builtin_nanf("");
        zf = 0.f;
    }
    z = (uint8_t)(int)zf;
#pragma unroll
    for (int i = 0; i < 2 * C; ++i) {
        const float u = fminf(fmaxf(rintf(x[i] / s) + zf, 0.f), most);
        code[i] = fine ? (uint8_t)(int)u : 0;
    }
}

// The blocks of 32 positions that hold new tokens of a sequence, dealt out over the workgroups:
// f(sequence, its rows, block, first and one past the last new token inside the block)
template <typename F>
__device__ inline void for_blocks(const CacheArgs &g, int nb, F &&f) {
    for (int64_t it = blockIdx.x; it < (int64_t)g.n_seq * nb; it += gridDim.x) {
        const int s = (int)(it / nb);
        const SeqRows r = seq_rows(g, s);
        const int end = (int)min((int64_t)r.past + r.n, (int64_t)g.cap);
        for (int blk = (r.past >> 5) + (int)(it % nb); blk * 32 < end; blk += nb) {
            const int t0 = max(r.past - blk * 32, 0), t1 = min(end - blk * 32, 32);
            if (t0 < t1) f(s, r, blk, t0, t1);
        }
    }
}

template <int DT, int DH, int BITS>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheArgs g, const void *__restrict__ yv, int64_t ldy, int nb) {
    typedef typename Mma<DT>::elem elem;
    constexpr int HALF = DH / 2, C = DH / 16, DHB = DH * BITS / 8;
    __shared__ double2 tab[32 * HALF];                 // (cos, sin) of the block's positions
    __shared__ __align__(16) uint8_t tile[DHB * PITCH];
    const int tid = threadIdx.x, e = tid & 7;
    const bool rope = g.freq[0] != 0.0, sym = g.k_zero == nullptr;
    for_blocks(g, nb, [&](int s, const SeqRows &r, int blk, int t0, int t1) {
        const int page = page_of(g, s, blk * 32);
        if (page < 0) return;
        const int nt = t1 - t0, at0 = (blk * 32) & ((1 << g.page_shift) - 1);
        if (rope) {
            __syncthreads();
            for (int i = tid; i < nt * HALF; i += 256) {
                double sn, cs;
                sincos((double)(blk * 32 + t0 + i / HALF) * g.freq[i % HALF], &sn, &cs);
                tab[i] = make_double2(cs, sn);
            }
            __syncthreads();
        }
        const elem *rows = static_cast<const elem *>(yv) + (int64_t)(r.row + (blk * 32 - r.past)) * ldy;
        // one (token, head): codes, key bytes and scales stored, value codes returned
        auto item = [&](int t, int h, uint8_t (&vc)[2 * C]) {
            const elem *kp = rows + (int64_t)t * ldy + (int64_t)(g.n_heads + h) * DH + e * C;
            const elem *vp = kp + (int64_t)g.n_kv_heads * DH;
            float x[2 * C], y[2 * C];
            load_c<DT, C>(kp, x);
            load_c<DT, C>(kp + HALF, x + C);
            load_c<DT, C>(vp, y);
            load_c<DT, C>(vp + HALF, y + C);
            if (rope) {
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    const double2 cs = tab[(t - t0) * HALF + e * C + i];
                    const double a = x[i], b = x[C + i];
                    x[i] = (float)(a * cs.x - b * cs.y);
                    x[C + i] = (float)(b * cs.x + a * cs.y);
                }
            }
            uint8_t kc[2 * C], kz, vz;
            float ks, vs;
            encode<BITS, C>(x, sym, kc, ks, kz);
            encode<BITS, C>(y, sym, vc, vs, vz);
            const int64_t slot = (((int64_t)page * g.n_kv_heads + h) << g.page_shift) + at0 + t;
            uint8_t *kr = g.k + slot * DHB + e * C;
            if constexpr (BITS == 8) {
                store_bytes<C>(kr, kc);
                store_bytes<C>(kr + HALF, kc + C);
            } else {
#pragma unroll
                for (int i = 0; i < C; ++i) {
                    kc[i] |= kc[C + i] << 4;
                    vc[i] |= vc[C + i] << 4;
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
            for (int i0 = 0; i0 < nt * g.n_kv_heads; i0 += 32) {
                const int i = i0 + (tid >> 3);
                if (i >= nt * g.n_kv_heads) break;     // eight lanes of an item leave together
                const int t = t0 + i % nt, h = i / nt;
                uint8_t vc[2 * C];
                item(t, h, vc);
                uint8_t *vb = vbase(h);
#pragma unroll
                for (int k = 0; k < NC; ++k) vb[(e * C + (k < C ? k : HALF + k - C)) * 32 + t] = vc[k];
            }
            return;
        }
        const int t = tid >> 3;
        for (int h = 0; h < g.n_kv_heads; ++h) {
            if (t >= t0 && t < t1) {
                uint8_t vc[2 * C];
                item(t, h, vc);
#pragma unroll
                for (int k = 0; k < NC; ++k) tile[(e * C + (k < C ? k : HALF + k - C)) * PITCH + t] = vc[k];
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
            __syncthreads();
        }
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
    for_blocks(g, nb, [&](int s, const SeqRows &r, int blk, int t0, int t1) {
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
            for (int i0 = 0; i0 < nt * g.n_kv_heads; i0 += 32) {
                const int i = i0 + (tid >> 3);
                if (i >= nt * g.n_kv_heads) break;
                const int t = t0 + i % nt, h = i / nt;
                const uint8_t *vb = vbase(h);
                item(t, h, [&](int d) { return vb[d * 32 + t]; });
            }
            return;
        }
        const int t = tid >> 3;
        for (int h = 0; h < g.n_kv_heads; ++h) {
            const uint8_t *vb = vbase(h);
            for (int c = tid; c < DHB * 2; c += 256) { // whole tiles: chunks of 16 tokens
                const u32x4 q = *reinterpret_cast<const u32x4 *>(vb + c * 16);
                uint2 *dst = reinterpret_cast<uint2 *>(tile + (c >> 1) * PITCH + (c & 1) * 16);
                dst[0] = make_uint2(q[0], q[1]);
                dst[1] = make_uint2(q[2], q[3]);
            }
            __syncthreads();
            if (t >= t0 && t < t1) item(t, h, [&](int d) { return tile[d * PITCH + t]; });
            __syncthreads();
        }
    });
}

// blocks of 32 positions that max_new tokens can touch, and the launch's workgroups (at most 2^20: a
// workgroup takes the next ones in turn)
int blocks_per_seq(const CacheArgs &g) { return (int)(((int64_t)g.max_new + 62) / 32); }
unsigned grid_of(const CacheArgs &g) {
    const int64_t n = (int64_t)g.n_seq * blocks_per_seq(g);
    return (unsigned)(n < (1 << 20) ? n : (1 << 20));
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
