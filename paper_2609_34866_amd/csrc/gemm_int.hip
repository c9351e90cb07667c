// gemm_int.hip -- the projection in 8-bit integers, and the row quantizer that feeds it.
//
// quant_rows: eq. quant's symmetric grid at 8 bits with one group per row: s = RN32(max|x| / 127) (1 if
// that is 0), code = clip(RNE(RN32(x / s)), -127, 127).
// project: y[m][n] = RN(RN32(acc) * RN32(sx[m] sw[n])), acc = sum_k xq[m][k] wq[n][k] in 32-bit integers:
// exact, so the result does not depend on the tile, the split or the order of the sum.
//
// Three kernels (launch_project_int chooses by the sizes):
//  * int_w4p_kernel: persistent, 256 x 256 tiles, one workgroup of four waves per CU, each wave 128 x 128 as 4 x 4
//    blocks of v_mfma_i32_32x32x32_i8; the LDS rings, refills and waits of gemm_w4p_kernel (gemm.hip), whose
//    16-byte chunks hold 16 codes here instead of 8 values, at twice the product rate per byte.
//  * int_small_kernel: 128 x 128 or 64 x 64 tiles for the shapes whose 256-tiles leave CUs idle.
//  * int_skinny_kernel: up to 32 tokens.  The weights are what is read: each wave streams 16, 32 or 64 weight
//    rows straight into registers, the waves of a workgroup share K, their sums meet in LDS.
#include <algorithm>

#include "device_common.h"
#include "kernels.h"
#include "lds_pipe.h"

namespace jab {
namespace {

typedef int i32x16 __attribute__((ext_vector_type(16)));

__device__ inline i32x16 mma_i8(i32x4 a, i32x4 b, i32x16 c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
}

template <int DT>
__device__ inline void load8f(const void *p, int64_t e, float *v) {
    if constexpr (DT == F32) {
        const f32x4 *q = reinterpret_cast<const f32x4 *>(static_cast<const float *>(p) + e);
        const f32x4 a = q[0], b = q[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = a[i];
            v[4 + i] = b[i];
        }
    } else {
        const u16x8 a = *reinterpret_cast<const u16x8 *>(static_cast<const uint16_t *>(p) + e);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f32<DT>(a[i]);
    }
}

// ---------------------------------------------------------------- row quantizer
// A workgroup of NT threads per row; a thread takes chunks of 8 values, NT chunks apart, the first CH of them
// kept in registers between the maximum and the codes (rows past NT * CH * 8 values are read again).
// |x| is compared as its bits without the sign, in which infinity and NaN lie above every finite
// value, so a row that holds one is found by its maximum: scale NaN, codes 0.
template <int DT, int NT, int CH>
__global__ __launch_bounds__(NT) void quant_rows_kernel(const void *__restrict__ src, int cols,
                                                        int8_t *__restrict__ codes, float *__restrict__ scale) {
    __shared__ uint32_t part[NT / 64];
    const int64_t row = blockIdx.x, e0 = row * cols;
    const int n = cols / 8;
    float v[CH][8];
    uint32_t mx = 0;
    auto upd = [&](const float *x) {
#pragma unroll
        for (int k = 0; k < 8; ++k) mx = max(mx, __builtin_bit_cast(uint32_t, x[k]) & 0x7FFFFFFFu);
    };
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = threadIdx.x + NT * i;
        if (c < n) {
            load8f<DT>(src, e0 + (int64_t)c * 8, v[i]);
            upd(v[i]);
        }
    }
    for (int c = threadIdx.x + NT * CH; c < n; c += NT) {
        float x[8];
        load8f<DT>(src, e0 + (int64_t)c * 8, x);
        upd(x);
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) mx = max(mx, (uint32_t)__shfl_xor((int)mx, off, 64));
    if constexpr (NT > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mx;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) mx = max(mx, part[i]);
    }
    const bool fine = mx < 0x7F800000u;
    // quotients as a division rounds them, without dividing: x times the fp64 reciprocal is within 2^-52 of x / s, which
    // is nearer than 2^-25 of its last place to no midpoint of two fp32 numbers, so both round alike
    float s = (float)((double)__builtin_bit_cast(float, mx) * (1.0 / 127));
    if (s == 0.f) s = 1.f;
    const double r = 1.0 / (double)s;
    const float most = fine ? 127.f : 0.f;                 // codes 0 where the scale is NaN
    if (threadIdx.x == 0) scale[row] = fine ? s : __builtin_nanf("");
    auto put = [&](int c, const float *x) {
        uint32_t o[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float u = __builtin_amdgcn_fmed3f(rintf((float)((double)x[k] * r)), -most, most);
            o[k >> 2] = __builtin_amdgcn_cvt_pk_u8_f32(u + 128.f, k & 3, o[k >> 2]);
        }
        *reinterpret_cast<uint2 *>(codes + e0 + (int64_t)c * 8) = make_uint2(o[0] ^ 0x80808080u, o[1] ^ 0x80808080u);
    };
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = threadIdx.x + NT * i;
        if (c < n) put(c, v[i]);
    }
    for (int c = threadIdx.x + NT * CH; c < n; c += NT) {
        float x[8];
        load8f<DT>(src, e0 + (int64_t)c * 8, x);
        put(c, x);
    }
}

// ---------------------------------------------------------------- product
struct IntArgs {
    const int8_t *A, *B;          // xq [M][K], wq [N][K]
    const float *sa, *sb;         // [M], [N]
    void *C;                      // [M][N] in the dtype
    int M, N, K;
    int tiles_m, tiles_n;
};

// row-dependent XOR key of the LDS rows' 16-byte chunks (CPR of them), so that the rows that one LDS cycle
// serves lie in distinct banks
template <int CPR>
__device__ inline int chunk_key(int r) {
    if constexpr (CPR == 8) return (r >> 1) & 7;
    else if constexpr (CPR == 4) return (r >> 2) & 3;
    else return (r >> 3) & 1;
}

// four consecutive outputs of a row from their sums: the row's scale, the columns' scales
__device__ inline f32x4 scaled4(int a0, int a1, int a2, int a3, float s, f32x4 t) {
    return f32x4{(float)a0 * (s * t[0]), (float)a1 * (s * t[1]), (float)a2 * (s * t[2]), (float)a3 * (s * t[3])};
}

// eight consecutive columns of a row per lane: the lane holds columns c .. c + 3 (a) and c + 8 .. c + 11 (b) of
// 16, c = 4 half; exchanging a of the upper half-wave with b of the lower one leaves 8 half .. 8 half + 7
template <int DT>
__device__ inline u32x4 join16(f32x4 a, f32x4 b) {
    uint32_t a0 = pack2<DT>(a[0], a[1]), a1 = pack2<DT>(a[2], a[3]);
    uint32_t b0 = pack2<DT>(b[0], b[1]), b1 = pack2<DT>(b[2], b[3]);
    asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\tv_permlane32_swap_b32 %2, %3\n\ts_nop 1"
                 : "+v"(a0), "+v"(b0), "+v"(a1), "+v"(b1));
    return u32x4{a0, a1, b0, b1};
}

// Tiles of BT x BT, four waves in a 2 x 2 arrangement; k-tiles of CPR chunks in a ring of NS stages, one
// barrier per k-tile (as gemm_small_kernel).  K a multiple of 16 CPR.
template <int DT, int BT, int CPR>
__global__ __launch_bounds__(256, 2) void int_small_kernel(IntArgs g) {
    typedef typename Mma<DT>::elem elem;
    constexpr int BK = CPR * 16, U = CPR / 2, FB = BT / 64;
    constexpr int ROWB = CPR * 16, PANEL = BT * ROWB, STAGE = 2 * PANEL;
    constexpr int NS = BT == 64 ? 3 : (65536 / STAGE < 4 ? 65536 / STAGE : 4);
    constexpr int DPP = BT * CPR / 256 > 0 ? BT * CPR / 256 : 1;    // DMA instructions per wave and panel
    constexpr int RPI = 64 / CPR;
    constexpr bool PART = BT * CPR < 256;                          // fewer DMA instructions than waves
    static_assert(NS >= 2, "ring");
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wr = wave >> 1, wc = wave & 1, half = lane >> 5, l32 = lane & 31;

    // XCD x takes a contiguous range of tiles, in groups of eight row tiles
    const int n_items = gridDim.x, x = blockIdx.x & 7;
    const int pid = x * (n_items >> 3) + min(x, n_items & 7) + (blockIdx.x >> 3);
    const int group_tiles = 8 * g.tiles_n, first_m = (pid / group_tiles) * 8, gsz = min(g.tiles_m - first_m, 8);
    const int bm0 = (first_m + (pid % group_tiles) % gsz) * BT, bn0 = (pid % group_tiles) / gsz * BT;
    const int nk = g.K / BK;
    const i32x4 rsA = buffer_rsrc(g.A + (int64_t)bm0 * g.K), rsB = buffer_rsrc(g.B + (int64_t)bn0 * g.K);
    uint32_t voffA[DPP], voffB[DPP];
#pragma unroll
    for (int i = 0; i < DPP; ++i) {
        // rows past an edge read the last row, for outputs that are not stored
        const int r = PART ? min(RPI * wave + lane / CPR, BT - 1) : RPI * (wave + 4 * i) + lane / CPR;
        const int c = (lane % CPR) ^ chunk_key<CPR>(r);
        voffA[i] = (uint32_t)(min(bm0 + r, g.M - 1) - bm0) * (uint32_t)g.K + c * 16;
        voffB[i] = (uint32_t)(min(bn0 + r, g.N - 1) - bn0) * (uint32_t)g.K + c * 16;
    }
    auto issue = [&](int kt, int slot) {      // k-tile kt (past the end: the last again, never read)
        const int kk = min(kt, nk - 1) * BK;
        unsigned char *st = smem + slot * STAGE;
        if (PART && RPI * wave >= BT) {       // this wave's share lies behind the panel: the first rows again
            buffer_dma16(rsA, voffA[0], kk, smem + NS * STAGE + wave * 1024);
            buffer_dma16(rsB, voffB[0], kk, smem + NS * STAGE + wave * 1024);
            return;
        }
#pragma unroll
        for (int i = 0; i < DPP; ++i) {
            buffer_dma16(rsA, voffA[i], kk, st + (wave + 4 * i) * 1024);
            buffer_dma16(rsB, voffB[i], kk, st + PANEL + (wave + 4 * i) * 1024);
        }
    };
    const int key = chunk_key<CPR>(l32);
    uint32_t rda[U], rdb[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int pc = (2 * u + half) ^ key;
        rda[u] = (uint32_t)((wr * (BT / 2) + l32) * ROWB + pc * 16);
        rdb[u] = (uint32_t)(PANEL + (wc * (BT / 2) + l32) * ROWB + pc * 16);
    }
    i32x16 acc[FB][FB];
#pragma unroll
    for (int i = 0; i < FB; ++i)
#pragma unroll
        for (int j = 0; j < FB; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    // the scales, not asked for at the end (4576 x 2304, K 768: 19.5 us with their loads there, 17.8)
    float sa[FB];
    f32x4 sb[FB][2][2];
#pragma unroll
    for (int i = 0; i < FB; ++i) {
        sa[i] = g.sa[min(bm0 + wr * (BT / 2) + 32 * i + l32, g.M - 1)];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int col = min(bn0 + wc * (BT / 2) + 32 * i + 16 * p, g.N - 16) + 4 * half;
            sb[i][p][0] = *reinterpret_cast<const f32x4 *>(g.sb + col);
            sb[i][p][1] = *reinterpret_cast<const f32x4 *>(g.sb + col + 8);
        }
    }
#pragma unroll
    for (int s0 = 0; s0 < NS - 1; ++s0) issue(s0, s0);
    int slot = 0;
    for (int kt = 0; kt < nk; ++kt) {
        wait_lgkm0();
        wait_vmcnt<(NS - 2) * 2 * DPP>();
        raw_barrier();
        issue(kt + NS - 1, slot == 0 ? NS - 1 : slot - 1);
        const unsigned char *st = smem + slot * STAGE;
        i32x4 fa[U][FB], fb[U][FB];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < FB; ++i) {
                fa[u][i] = *reinterpret_cast<const i32x4 *>(st + rda[u] + i * 32 * ROWB);
                fb[u][i] = *reinterpret_cast<const i32x4 *>(st + rdb[u] + i * 32 * ROWB);
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < FB; ++i)
#pragma unroll
                for (int j = 0; j < FB; ++j) acc[i][j] = mma_i8(fb[u][j], fa[u][i], acc[i][j]);
        slot = slot == NS - 1 ? 0 : slot + 1;
    }
    wait_vmcnt<0>();
    // acc[i][j][4 q + t] = sum of row 32 i + l32, column 32 j + 8 q + 4 half + t (wave's quarter); N is a
    // multiple of 16, so 16 columns are inside or outside as a whole
#pragma unroll
    for (int i = 0; i < FB; ++i) {
        const int row = bm0 + wr * (BT / 2) + 32 * i + l32;
        if (row >= g.M) continue;
        const float s = sa[i];
        elem *crow = static_cast<elem *>(g.C) + (int64_t)row * g.N;
#pragma unroll
        for (int j = 0; j < FB; ++j)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int col = bn0 + wc * (BT / 2) + 32 * j + 16 * p;
                if (col >= g.N) continue;
                const f32x4 ta = sb[j][p][0], tb = sb[j][p][1];
                const i32x16 &d = acc[i][j];
                const f32x4 a = scaled4(d[8 * p], d[8 * p + 1], d[8 * p + 2], d[8 * p + 3], s, ta);
                const f32x4 b = scaled4(d[8 * p + 4], d[8 * p + 5], d[8 * p + 6], d[8 * p + 7], s, tb);
                if constexpr (DT == F32) {
                    *reinterpret_cast<f32x4 *>(crow + col + 4 * half) = a;
                    *reinterpret_cast<f32x4 *>(crow + col + 8 + 4 * half) = b;
                } else {
                    *reinterpret_cast<u32x4 *>(crow + col + 8 * half) = join16<DT>(a, b);
                }
            }
    }
}

// The persistent kernel: gemm_w4p_kernel's schedule (three k-tiles of the tokens and two of the weights in
// 160 KiB of LDS, refills one DMA instruction every fourth product, one barrier per k-tile, the rings running on
// across tiles) with k-tiles of 128 codes.  Needs M, N >= 256, K a multiple of 128 and at least 384.
template <int DT>
__global__ __launch_bounds__(256, 1) void int_w4p_kernel(IntArgs g) {
    typedef typename Mma<DT>::elem elem;
    constexpr int CPR = 8, BK = 128, U = 4, ROWB = 128, HALF = 256 * ROWB, DPA = 8, RPI = 8;
    constexpr int ABASE = 0, BBASE = 3 * HALF;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wr = wave >> 1, wc = wave & 1, half = lane >> 5, l32 = lane & 31;
    const int nk = g.K / BK, n_work = g.tiles_m * g.tiles_n;

    struct Tile {
        int bm0, bn0;
        i32x4 rsA, rsB;
    };
    // work item -> tile: each XCD a contiguous range, in groups of eight row tiles; the last tile of a
    // ragged direction is moved back to end at the edge (what it shares with its neighbour is
    // written twice with the same values: integer sums)
    auto decode = [&](int work, Tile &t) {
        int pid = work;
        if ((n_work & 7) == 0) pid = (pid & 7) * (n_work >> 3) + (pid >> 3);
        const int group_tiles = 8 * g.tiles_n, first_m = (pid / group_tiles) * 8, gsz = min(g.tiles_m - first_m, 8);
        t.bm0 = min((first_m + (pid % group_tiles) % gsz) * 256, g.M - 256);
        t.bn0 = min((pid % group_tiles) / gsz * 256, g.N - 256);
        t.rsA = buffer_rsrc(g.A + (int64_t)t.bm0 * g.K);
        t.rsB = buffer_rsrc(g.B + (int64_t)t.bn0 * g.K);
    };
    // DMA instruction i of an operand: rows RPI (wave + 4 i) .. + RPI - 1, whose chunk key does not depend on i
    const int r0 = RPI * wave + lane / CPR;
    const uint32_t voff0 = (uint32_t)r0 * (uint32_t)g.K + (((lane % CPR) ^ chunk_key<CPR>(r0)) * 16);
    uint32_t voff[DPA];
#pragma unroll
    for (int i = 0; i < DPA; ++i) voff[i] = voff0 + (uint32_t)(32 * i) * (uint32_t)g.K;
    auto issueA = [&](const Tile &t, int i, int kt, int slot) {
        buffer_dma16(t.rsA, voff[i], kt * BK, smem + ABASE + slot * HALF + (wave + 4 * i) * 1024);
    };
    auto issueB = [&](const Tile &t, int i, int kt, int slot) {
        buffer_dma16(t.rsB, voff[i], kt * BK, smem + BBASE + slot * HALF + (wave + 4 * i) * 1024);
    };
    const int key = chunk_key<CPR>(l32);
    uint32_t rda[U], rdb[U];
#pragma unroll
    for (int ks = 0; ks < U; ++ks) {
        const int pc = (2 * ks + half) ^ key;
        rda[ks] = (uint32_t)((wr * 128 + l32) * ROWB + pc * 16);
        rdb[ks] = (uint32_t)((wc * 128 + l32) * ROWB + pc * 16);
    }
    i32x4 fa[2][4], fb[2][4];
    auto rd = [&](int r, int da, int sb, int ks, int buf) {
        const unsigned char *ab = smem + ABASE + da * HALF, *bb = smem + BBASE + sb * HALF;
        if (r == 0) fa[buf][0] = *(const i32x4 *)(ab + rda[ks]);
        else if (r <= 4) fb[buf][r - 1] = *(const i32x4 *)(bb + rdb[ks] + (r - 1) * 32 * ROWB);
        else fa[buf][r - 4] = *(const i32x4 *)(ab + rda[ks] + (r - 4) * 32 * ROWB);
    };
    int work = blockIdx.x;
    if (work >= n_work) return;
    Tile cur, nxt;
    decode(work, cur);
    bool has_next = work + (int)gridDim.x < n_work;
    if (has_next) decode(work + gridDim.x, nxt);
    else nxt = cur;                                   // the refills re-load its first k-tiles (never read)

    // prologue, as a previous tile's last stages leave the rings
#pragma unroll
    for (int i = 0; i < DPA; ++i) issueA(cur, i, 0, 0);
#pragma unroll
    for (int i = 0; i < DPA; ++i) issueB(cur, i, 0, 0);
#pragma unroll
    for (int i = 0; i < DPA; ++i) issueA(cur, i, 1, 1);
#pragma unroll
    for (int i = 0; i < DPA / 2; ++i) issueB(cur, i, 1, 1);
    wait_vmcnt<DPA + DPA / 2>();
    raw_barrier();
#pragma unroll
    for (int r = 0; r < 8; ++r) rd(r, 0, 0, 0, 0);

    i32x16 acc[4][4];
    int da = 0, sb = 0;                               // the stage's slots of the deep (A) and shallow (B) ring
    for (;;) {
        // Stage kt: per k-step 16 products, a fragment read of the next k-step every other product; refills of
        // the shallow ring's second half of k-tile kt + 1 in k-step 0, of the deep ring's k-tile kt + 2 in k-steps
        // 1 and 2, of the shallow ring's first half of k-tile kt + 2 after the barrier; the barrier before the last
        // k-step waits for k-tile kt + 1 and leaves the 8 deep loads of kt + 2 in flight
        auto stage = [&](int kt, auto first_c) {
            constexpr bool FIRST = decltype(first_c)::value;
            const int nd = da == 2 ? 0 : da + 1, ns = sb ^ 1, rd_ = da == 0 ? 2 : da - 1;
            const bool n2 = kt + 2 >= nk, n1 = kt + 1 >= nk;
            const Tile &t2 = n2 ? nxt : cur;
            const Tile &t1 = n1 ? nxt : cur;
            const int k2 = n2 ? kt + 2 - nk : kt + 2, k1 = n1 ? kt + 1 - nk : kt + 1;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int cb = u & 1;
                if (u == U - 1) {
                    wait_lgkm0();
                    wait_vmcnt<DPA>();
                    raw_barrier();
                }
#pragma unroll
                for (int m = 0; m < 16; ++m) {
                    const int i = m >> 2, j = m & 3;
                    if (FIRST && u == 0) acc[i][j] = mma_i8(fb[cb][j], fa[cb][i], i32x16{});
                    else acc[i][j] = mma_i8(fb[cb][j], fa[cb][i], acc[i][j]);
                    if ((m & 1) == 0) {
                        if (u < U - 1) rd(m >> 1, da, sb, u + 1, cb ^ 1);
                        else rd(m >> 1, nd, ns, 0, cb ^ 1);
                    }
                    if ((m & 3) == 0) {
                        if (u == 0) issueB(t1, DPA / 2 + (m >> 2), k1, ns);
                        else if (u <= 2) issueA(t2, 4 * (u - 1) + (m >> 2), k2, rd_);
                        else issueB(t2, m >> 2, k2, sb);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            da = nd;
            sb = ns;
        };
        stage(0, std::integral_constant<bool, true>());
        for (int kt = 1; kt < nk; ++kt) stage(kt, std::integral_constant<bool, false>());

        // epilogue from registers: acc[i][j][4 q + t] = sum of row wr*128 + 32 i + l32, column wc*128 + 32 j +
        // 8 q + 4 half + t; accumulators are read one block at a time
        f32x4 tw[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                tw[j][q] = *reinterpret_cast<const f32x4 *>(g.sb + cur.bn0 + wc * 128 + 32 * j + 8 * q + 4 * half);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = cur.bm0 + wr * 128 + 32 * i + l32;
            const float s = g.sa[row];
            elem *crow = static_cast<elem *>(g.C) + (int64_t)row * g.N;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int colb = cur.bn0 + wc * 128 + 32 * j;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    int v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v[e]) : "a"(acc[i][j][8 * p + e]));
                    const f32x4 a = scaled4(v[0], v[1], v[2], v[3], s, tw[j][2 * p]);
                    const f32x4 b = scaled4(v[4], v[5], v[6], v[7], s, tw[j][2 * p + 1]);
                    if constexpr (DT == F32) {
                        *reinterpret_cast<f32x4 *>(crow + colb + 16 * p + 4 * half) = a;
                        *reinterpret_cast<f32x4 *>(crow + colb + 16 * p + 8 + 4 * half) = b;
                    } else {
                        *reinterpret_cast<u32x4 *>(crow + colb + 16 * p + 8 * half) = join16<DT>(a, b);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        if (!has_next) break;
        cur = nxt;
        work += gridDim.x;
        has_next = work + (int)gridDim.x < n_work;
        if (has_next) decode(work + gridDim.x, nxt);
    }
    wait_vmcnt<0>();
}

// Few tokens: a workgroup takes 16 RT weight rows and all tokens (16 MT), its eight waves each an eighth of K (in steps of
// 64 codes: v_mfma_i32_16x16x64_i8, lane (row l % 16, g = l / 16) holding codes 16 g .. 16 g + 15 of the step).  Weights
// and tokens go from memory to registers, UNR steps at once; the sums of the waves meet in LDS.  Bound by the bytes
// that a CU takes in: every workgroup reads all tokens' codes over.  24 tokens, 6144 rows, K 4096 (25 MB of weights):
// 12.5 us with RT 1, 9.9 with the 2 that the rule takes; a device copy of as many bytes takes 7.7.  More steps at once, nontemporal
// loads or another order of the steps changed nothing.
constexpr int SK_WAVES = 8;
template <int DT, int RT, int MT>
__global__ __launch_bounds__(64 * SK_WAVES) void int_skinny_kernel(IntArgs g) {
    typedef typename Mma<DT>::elem elem;
    static_assert(RT * MT <= SK_WAVES, "one wave per tile at the end");
    constexpr int UNR = RT * MT == 8 ? 2 : 4;
    __shared__ i32x4 red[SK_WAVES][RT * MT][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int l16 = lane & 15, grp = lane >> 4;
    const int n0 = blockIdx.x * 16 * RT;
    const int steps = (g.K + 63) / 64;
    const int s0 = (int)((int64_t)steps * wave / SK_WAVES), s1 = (int)((int64_t)steps * (wave + 1) / SK_WAVES);
    const int8_t *wp[RT], *xp[MT];
#pragma unroll
    for (int r = 0; r < RT; ++r) wp[r] = g.B + (int64_t)min(n0 + 16 * r + l16, g.N - 1) * g.K + grp * 16;
#pragma unroll
    for (int t = 0; t < MT; ++t) xp[t] = g.A + (int64_t)min(16 * t + l16, g.M - 1) * g.K + grp * 16;
    i32x4 acc[RT][MT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[r][t] = i32x4{0, 0, 0, 0};
    for (int s = s0; s < s1; s += UNR) {
        i32x4 w[UNR][RT], x[UNR][MT];
#pragma unroll
        for (int u = 0; u < UNR; ++u) {
            const int k = 64 * (s + u);
            // past the wave's share, or the last 32 of a K that is no multiple of 64: zeros for the weights
            // (any codes for the tokens)
            const bool in = s + u < s1 && k + 16 * grp < g.K;
            const int at = in ? k : -16 * grp;
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                w[u][r] = *reinterpret_cast<const i32x4 *>(wp[r] + at);
                if (!in) w[u][r] = i32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int t = 0; t < MT; ++t) x[u][t] = *reinterpret_cast<const i32x4 *>(xp[t] + at);
        }
#pragma unroll
        for (int u = 0; u < UNR; ++u)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    acc[r][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u][r], x[u][t], acc[r][t], 0, 0, 0);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < MT; ++t) red[wave][r * MT + t][lane] = acc[r][t];
    __syncthreads();
    // acc[r][t][i]: token 16 t + l16, weight row n0 + 16 r + 4 grp + i
    if (wave < RT * MT) {
        i32x4 s = red[0][wave][lane];
#pragma unroll
        for (int w = 1; w < SK_WAVES; ++w) {
            const i32x4 v = red[w][wave][lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += v[e];
        }
        const int m = 16 * (wave % MT) + l16, n = n0 + 16 * (wave / MT) + 4 * grp;
        if (m < g.M && n < g.N) {
            const f32x4 o = scaled4(s[0], s[1], s[2], s[3], g.sa[m], *reinterpret_cast<const f32x4 *>(g.sb + n));
            elem *c = static_cast<elem *>(g.C) + (int64_t)m * g.N + n;
            if constexpr (DT == F32) *reinterpret_cast<f32x4 *>(c) = o;
            else *reinterpret_cast<uint2 *>(c) = make_uint2(pack2<DT>(o[0], o[1]), pack2<DT>(o[2], o[3]));
        }
    }
}

constexpr int CUS = 256;

template <int DT, int BT, int CPR>
hipError_t run_small(IntArgs a, hipStream_t st) {
    constexpr int STAGE = 2 * BT * CPR * 16;
    constexpr int NS = BT == 64 ? 3 : (65536 / STAGE < 4 ? 65536 / STAGE : 4);
    constexpr size_t LDS = (size_t)NS * STAGE + (BT * CPR < 256 ? 4096 : 0);
    a.tiles_m = (a.M + BT - 1) / BT;
    a.tiles_n = (a.N + BT - 1) / BT;
    hipError_t e = hipFuncSetAttribute((const void *)int_small_kernel<DT, BT, CPR>,
                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)LDS);
    if (e != hipSuccess) return e;
    int_small_kernel<DT, BT, CPR><<<dim3(a.tiles_m * a.tiles_n), 256, LDS, st>>>(a);
    return hipGetLastError();
}

// The weight rows of a workgroup: what a CU takes in is, per workgroup that it gets, RT + MT tiles of 16 rows; the RT
// with the least of it.
template <int DT, int MT>
hipError_t run_skinny(IntArgs a, hipStream_t st) {
    const int tiles = (a.N + 15) / 16;
    auto groups = [&](int rt) { return (tiles + rt - 1) / rt; };
    auto cost = [&](int rt) { return (int64_t)((groups(rt) + CUS - 1) / CUS) * (rt + MT); };
    int rt = cost(2) < cost(1) ? 2 : 1;
    if (cost(4) < cost(rt)) rt = 4;
    if (rt == 1) int_skinny_kernel<DT, 1, MT><<<groups(1), 64 * SK_WAVES, 0, st>>>(a);
    else if (rt == 2) int_skinny_kernel<DT, 2, MT><<<groups(2), 64 * SK_WAVES, 0, st>>>(a);
    else int_skinny_kernel<DT, 4, MT><<<groups(4), 64 * SK_WAVES, 0, st>>>(a);
    return hipGetLastError();
}

template <int DT>
hipError_t run_int(IntArgs a, hipStream_t st) {
    // Few tokens where 64-tiles leave CUs idle (bf16; this / 64-tiles): 1 token 6144 x 4096 7.0 / 10.9 us, 24 tokens 9.6 / 10.9,
    // 6144 x 16384 30 / 34; not 64 tokens (14.3 / 11.1), 32 of 2304 x 768 (5.2 / 4.5), 32 of 24576 x 4096 (26 / 17.5)
    if ((a.N + 63) / 64 <= CUS) {
        if (a.M <= 16) return run_skinny<DT, 1>(a, st);
        if (a.M <= 32 && a.K >= 1024) return run_skinny<DT, 2>(a, st);
    }
    const int64_t tm = (a.M + 255) / 256, tn = (a.N + 255) / 256, t = tm * tn;
    // the 256-tiles where they fill their rounds of one workgroup per CU to at least 60 % (bf16, K 4096; 128-tiles / these:
    // 66 % 57.9 / 52.6 and 105 / 97.5 us, 75 % 63.6 / 61.8, 94 % 77.5 / 58.7; but 47 % 38.0 / 47.2, and 56 % at K 1024 30.6 / 34.4)
    if (a.M >= 256 && a.N >= 256 && a.K % 128 == 0 && a.K >= 1024 && 10 * t >= 6 * ((t + CUS - 1) / CUS) * CUS) {
        constexpr size_t LDS = 5 * 256 * 128;
        a.tiles_m = (int)tm;
        a.tiles_n = (int)tn;
        hipError_t e = hipFuncSetAttribute((const void *)int_w4p_kernel<DT>,
                                           hipFuncAttributeMaxDynamicSharedMemorySize, (int)LDS);
        if (e != hipSuccess) return e;
        int_w4p_kernel<DT><<<dim3((unsigned)std::min<int64_t>(t, CUS)), 256, LDS, st>>>(a);
        return hipGetLastError();
    }
    // 128-tiles where they occupy three quarters of the CUs (K 4096; 64-tiles / these: 96 tiles 14.9 / 21.6 us, 192 24.5 / 24.0,
    // 240 30.3 / 24.7, 384 43.2 / 34.5)
    const bool big = (int64_t)((a.M + 127) / 128) * ((a.N + 127) / 128) >= CUS * 3 / 4;
    if (a.K % 128 == 0) return big ? run_small<DT, 128, 8>(a, st) : run_small<DT, 64, 8>(a, st);
    if (a.K % 64 == 0) return big ? run_small<DT, 128, 4>(a, st) : run_small<DT, 64, 4>(a, st);
    return big ? run_small<DT, 128, 2>(a, st) : run_small<DT, 64, 2>(a, st);
}

constexpr int64_t MOST_GROUPS = 1 << 23;              // workgroups of one launch (a grid has below 2^32 threads)

template <int DT>
hipError_t run_quant_rows(int64_t rows, int cols, const void *src, int8_t *codes, float *scale, hipStream_t st) {
    for (int64_t r = 0; r < rows; r += MOST_GROUPS) {
        const dim3 grid((unsigned)std::min(rows - r, MOST_GROUPS));
        const void *x = static_cast<const typename Mma<DT>::elem *>(src) + r * cols;
        // eight elements a thread; 4576 rows of 768 fp16: 6.0 us with 128 threads, 7.4 with 256, 6.2 with 64 twice; 24 rows
        // of 4096 bf16 (twice with 256): 3.4 us, 4.4 with 128 four times, 3.3 with 512; 32768: 71, 78 and 83 us (5.7 TB/s)
        if (cols <= 512) quant_rows_kernel<DT, 64, 1><<<grid, 64, 0, st>>>(x, cols, codes + r * cols, scale + r);
        else if (cols <= 1024) quant_rows_kernel<DT, 128, 1><<<grid, 128, 0, st>>>(x, cols, codes + r * cols, scale + r);
        else quant_rows_kernel<DT, 256, 2><<<grid, 256, 0, st>>>(x, cols, codes + r * cols, scale + r);
    }
    return hipGetLastError();
}

// a launch takes as many rows as its smallest tiles' workgroups allow
template <int DT>
hipError_t run_rows(IntArgs a, hipStream_t st) {
    const int64_t most = std::max<int64_t>(1, MOST_GROUPS / ((a.N + 63) / 64)) * 64, M = a.M;
    typename Mma<DT>::elem *C = static_cast<typename Mma<DT>::elem *>(a.C);
    const int8_t *A = a.A;
    const float *sa = a.sa;
    for (int64_t m = 0; m < M; m += most) {
        a.A = A + m * a.K;
        a.sa = sa + m;
        a.C = C + m * a.N;
        a.M = (int)std::min(M - m, most);
        const hipError_t e = run_int<DT>(a, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
}  // namespace

hipError_t launch_quant_rows(int dtype, int64_t rows, int cols, const void *src, int8_t *codes, float *scale,
                             hipStream_t st) {
    switch (dtype) {
    case F32: return run_quant_rows<F32>(rows, cols, src, codes, scale, st);
    case F16: return run_quant_rows<F16>(rows, cols, src, codes, scale, st);
    default: return run_quant_rows<BF16>(rows, cols, src, codes, scale, st);
    }
}

hipError_t launch_project_int(int dtype, const int8_t *xq, const float *sx, const int8_t *wq, const float *sw, void *y,
                              int M, int N, int K, hipStream_t st) {
    IntArgs a{xq, wq, sx, sw, y, M, N, K, 0, 0};
    switch (dtype) {
    case F32: return run_rows<F32>(a, st);
    case F16: return run_rows<F16>(a, st);
    default: return run_rows<BF16>(a, st);
    }
}

}  // namespace jab
