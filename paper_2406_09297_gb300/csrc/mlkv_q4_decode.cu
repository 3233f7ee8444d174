// Single-token decode attention over the 4-bit KV cache (layout and values: mlkv_q4.h), with an
// optional sliding window and sinks (MLKV, arXiv 2406.09297, Sec. 3; attention of Eqs. 2-3).
//
//   out = sum_t p_t v_t / sum_t p_t,  p_t = 2^(log2(e) q.k_t / sqrt(D) - m),  k_t = s_t (c_t - 8)
//
// per group of 32 channels.  K and V are never widened: a word's nibbles become bf16 128 + c by one
// mask-or each (the code's bits in the mantissa), which mma.m16n8k16 takes as its A operand straight
// from registers (16 positions or 16 channels by 8 query heads).  The surplus of 136 a channel goes
// into the accumulator it starts from:
//   S:  acc = -136 sum_c q_c + sum_c (128 + c_tc) q_c, exact products, at most 32 terms; the group's
//       scale multiplies the finished sum in fp32.
//   O:  P'_t = bf16(p_t s_t) per group is the B operand; acc = -136 sum_t P'_t (an MMA with -136s for
//       A, the same rounded P') + sum_t (128 + c_tc) P'_t over one tile, then added to O in fp32.
// p is rounded to bf16 once for the transposition and the sum of weights, and once more with the
// scale; both errors are relative, independent from position to position, and average out as the
// bf16 weights of the other decode kernel do.
//
// Work split as in decode_kernel: the tiles of all (sequence, KV head) segments end to end, an equal run
// of them for each persistent CTA; a CTA's warps take its tiles in turn, each through a ring of its own
// (one bulk copy a tile: a block's codes and scales lie together), so nothing but the ends of
// segments makes warps wait for one another.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "mlkv_q4.h"

#include "mlkv_device.cuh"

namespace mlkv {
namespace {

template <int D, int NB>
struct Q4Plan {
    using LY = Q4Layout<D>;
    static constexpr int kWarps = 8;
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kT = q4_tile_tokens(D);
    static constexpr int kSub = kT / kQ4Block;                  // blocks of a tile
    static constexpr int kStages = 2;
    static constexpr int kTileBytes = kSub * LY::kBytes;
    static constexpr int kMinBlocks = 2;
    static constexpr int kRing = 0;                             // [kWarps][kStages]
    // A piece's sums of 8 heads from every warp; rows padded so that the fragments' 16-byte stores
    // fall in distinct banks.
    static constexpr int kRow = D + 4;
    static constexpr int kRaw = kRing + kWarps * kStages * kTileBytes;
    static constexpr int kStat = kRaw + kWarps * 8 * kRow * 4;  // m, l [8 NB heads][kWarps] each
    // The piece's queries, rows padded so that a quarter warp's 16-byte loads fall in distinct
    // banks, and -136 times their group sums [group][16 heads].
    static constexpr int kQRow = D * 2 + 64;
    static constexpr int kQ = kStat + 2 * 8 * NB * kWarps * 4;
    static constexpr int kBias = kQ + 8 * NB * kQRow;
    static constexpr int kFlags = kBias + LY::kGroups * 16 * 4;
    static constexpr int kBars = kFlags + 16;
    static constexpr int kBytes = kBars + kWarps * kStages * 8;
    static_assert(kMinBlocks * (kBytes + 1024) <= 228 * 1024, "shared memory of the resident CTAs");
    static_assert(kTileBytes % 128 == 0 && kRaw % 16 == 0 && kQ % 16 == 0 && kBars % 8 == 0, "");
};

// A (sequence, KV head) segment as the walk sees it.
struct Segment {
    int beta, j, L;
    int first;            // its first tile in the flattened list
    VisibleTiles v;
};

template <int T>
__device__ __forceinline__ void load_segment(const Q4DecodeParams &p, Segment &s)
{
    s.L = p.uniform_len > 0 ? p.uniform_len : p.seq_len[s.beta];
    s.v = visible_tiles(s.L, p.window, p.sinks, T, kQ4Block);
}

template <int T>
__device__ __forceinline__ Segment segment_of_tile(const Q4DecodeParams &p, int tile)
{
    Segment s;
    if (p.uniform_len > 0) {
        s.beta = 0;
        load_segment<T>(p, s);
        const int seg = tile / s.v.nt;
        s.beta = seg / p.g;
        s.j = seg - s.beta * p.g;
        s.first = seg * s.v.nt;
        return s;
    }
    int lo = 0, hi = p.b - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.tile_start[mid] <= tile)
            lo = mid;
        else
            hi = mid - 1;
    }
    s.beta = lo;
    load_segment<T>(p, s);
    s.j = (tile - p.tile_start[lo]) / s.v.nt;
    s.first = p.tile_start[lo] + s.j * s.v.nt;
    return s;
}

template <int T>
__device__ __forceinline__ void next_segment(const Q4DecodeParams &p, Segment &s)
{
    s.first += s.v.nt;
    if (++s.j == p.g) {
        s.j = 0;
        if (++s.beta < p.b && p.uniform_len <= 0)
            load_segment<T>(p, s);
    }
}

// First position of tile tt, and the end of what is visible from there on.
template <int T>
__device__ __forceinline__ void tile_range(const Segment &s, int sinks, int tt, int &pos0, int &end)
{
    const bool sink = tt < s.v.ns;
    pos0 = tt * T + (sink ? 0 : s.v.skip);
    end = sink ? sinks : s.L;
}

// D = A B + C with its own registers for D.
__device__ __forceinline__ void mma_from(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1, float c0, float c1,
                                         float c2, float c3)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 "
        "{%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}

__device__ __forceinline__ uint32_t hmul2_bf16(uint32_t a, uint32_t b)
{
    const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162 *>(&a);
    const __nv_bfloat162 y = *reinterpret_cast<const __nv_bfloat162 *>(&b);
    const __nv_bfloat162 z = __hmul2(x, y);
    return *reinterpret_cast<const uint32_t *>(&z);
}

// Nibbles i and i + 4 of a word as the bf16 pair 128 + code.
__device__ __forceinline__ uint32_t codes_at(uint32_t w, int i)
{
    return ((w >> (4 * i)) & 0x000f000fu) | 0x43004300u;
}

// Reference maxima move when a score exceeds them by more than this (log2 units): weights stay <= 2^8.
constexpr float kQ4LazyMax = 8.f;
constexpr uint32_t kOnes2 = 0x3f803f80u;
constexpr uint32_t kMinus136 = 0xc308c308u;

template <int D, int NB>
__global__ void __launch_bounds__(Q4Plan<D, NB>::kThreads, Q4Plan<D, NB>::kMinBlocks)
    q4_decode_kernel(const __grid_constant__ Q4DecodeParams p)
{
    using PL = Q4Plan<D, NB>;
    using LY = Q4Layout<D>;
    constexpr int NW = PL::kWarps, T = PL::kT, NS = PL::kSub, NG = LY::kGroups, R = PL::kStages;
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t sbase = smem_addr(smem);
    volatile int *flags = reinterpret_cast<volatile int *>(smem + PL::kFlags);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int gid = lane >> 2, tig = lane & 3;
    const int P = gridDim.x, cta = blockIdx.x, N = p.num_tiles;
    const int tile_lo = static_cast<int>(static_cast<long long>(cta) * N / P);
    const int tile_hi = static_cast<int>(static_cast<long long>(cta + 1) * N / P);
    const uint32_t ring = sbase + PL::kRing + warp * R * PL::kTileBytes;
    const uint32_t bar_full = sbase + PL::kBars + warp * R * 8;
    const float NEG_INF = -__int_as_float(0x7f800000);
    if (lane == 0) {
        for (int s = 0; s < R; ++s)
            mbar_init(bar_full + 8 * s, 1);
        if (warp == 0)
            flags[0] = 0;
        fence_barrier_init();
    }
    __syncwarp();

    // The warp's tiles: tile_lo + warp, + NW, ...  Lane 0 sends each tile's copy R tiles ahead.
    Segment fs = segment_of_tile<T>(p, tile_lo < N ? tile_lo : N - 1);
    int f_tile = tile_lo + warp, f_it = 0;
    auto fetch = [&]() {
        if (f_tile >= tile_hi)
            return;
        while (f_tile >= fs.first + fs.v.nt)
            next_segment<T>(p, fs);
        if (lane == 0) {
            int pos0, end;
            tile_range<T>(fs, p.sinks, f_tile - fs.first, pos0, end);
            const int n = min(NS, (end - pos0 + kQ4Block - 1) / kQ4Block);
            const uint32_t bytes = static_cast<uint32_t>(n) * LY::kBytes;
            const uint32_t bar = bar_full + 8 * (f_it % R);
            mbar_arrive_expect_tx(bar, bytes);
            bulk_load(ring + (f_it % R) * PL::kTileBytes,
                      p.slot + (static_cast<long long>(fs.beta) * p.g + fs.j) * p.row_bytes +
                          static_cast<long long>(pos0 / kQ4Block) * LY::kBytes,
                      bytes, bar);
        }
        f_tile += NW;
        ++f_it;
    };
    // Queries of a segment: 16 bytes a thread; and the sums of their groups (four neighbours each).
    constexpr int kQThreads = 8 * NB * (D / 8);
    static_assert(kQThreads <= PL::kThreads, "one load a thread");
    auto load_q = [&](const Segment &s) {
        const int head = tid / (D / 8);
        uint4 v = make_uint4(0, 0, 0, 0);
        if (tid < kQThreads && head < p.G)
            v = *reinterpret_cast<const uint4 *>(
                p.Q + (static_cast<size_t>(s.beta) * p.h + static_cast<size_t>(s.j) * p.G) * D +
                tid * 8);
        return v;
    };
    auto store_q = [&](const uint4 &v) {
        const int head = tid / (D / 8), oct = tid % (D / 8);
        float sum = (bf16_lo(v.x) + bf16_hi(v.x)) + (bf16_lo(v.y) + bf16_hi(v.y)) +
                    ((bf16_lo(v.z) + bf16_hi(v.z)) + (bf16_lo(v.w) + bf16_hi(v.w)));
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if (tid < kQThreads) {
            *reinterpret_cast<uint4 *>(smem + PL::kQ + head * PL::kQRow + oct * 16) = v;
            if ((oct & 3) == 0)
                reinterpret_cast<float *>(smem + PL::kBias)[(oct >> 2) * 16 + head] = -136.f * sum;
        }
    };

    grid_dependency_wait();
    grid_dependents_launch();
    if (tile_lo >= tile_hi)
        return;
    Segment cs = segment_of_tile<T>(p, tile_lo);
#pragma unroll
    for (int s = 0; s < R; ++s)
        fetch();
    store_q(load_q(cs));
    __syncthreads();

    int it = 0;                       // this warp's tiles so far
    int tile = tile_lo + warp;
    for (int piece = tile_lo; piece < tile_hi;) {
        const int seg_end = cs.first + cs.v.nt;
        const int piece_end = min(seg_end, tile_hi);
        const bool last = piece_end == tile_hi;
        // the next piece's queries travel while this one is computed
        Segment ns = cs;
        uint4 q_next = make_uint4(0, 0, 0, 0);
        if (!last) {
            next_segment<T>(p, ns);
            q_next = load_q(ns);
        }
        float o[NB][2 * NG][4];
        float la[NB][4], m_run[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int n = 0; n < 2 * NG; ++n)
                o[nb][n][0] = o[nb][n][1] = o[nb][n][2] = o[nb][n][3] = 0.f;
            la[nb][0] = la[nb][1] = la[nb][2] = la[nb][3] = 0.f;
            m_run[nb][0] = m_run[nb][1] = NEG_INF;
        }
        for (; tile < piece_end; tile += NW, ++it) {
            const int s = it % R;
            int ok = 1;
            if (!mbar_wait(bar_full + 8 * s, (it / R) & 1)) {
                ok = 0;
                flags[0] = 1;
                atomicOr(p.err, kErrWaitFull);
            }
            const uint8_t *st = smem + PL::kRing + (warp * R + s) * PL::kTileBytes;
            int pos0, end;
            tile_range<T>(cs, p.sinks, tile - cs.first, pos0, end);
            const int vis0 = (tile - cs.first < cs.v.ns ? 0 : cs.v.first) - pos0;   // visible: [vis0, vis1)
            const int vis1 = end - pos0;
            const bool edge = vis0 > 0 || vis1 < T;
            if (__all_sync(0xffffffffu, ok)) {
                // ---- S = K Q^T, 16 positions by 8 heads a block ----
                float sc[NS][NB][4];
                uint32_t kw[NS][2 * NG];       // [hi][group]
                uint32_t kss[NS][NG];          // the scales of rows gid, gid + 8: group pairs
#pragma unroll
                for (int b = 0; b < NS; ++b) {
                    const uint8_t *blk = st + b * LY::kBytes;
#pragma unroll
                    for (int q = 0; q < 2 * NG / 4; ++q) {
                        const uint4 w = *reinterpret_cast<const uint4 *>(blk + q * 512 + lane * 16);
                        kw[b][4 * q] = w.x;
                        kw[b][4 * q + 1] = w.y;
                        kw[b][4 * q + 2] = w.z;
                        kw[b][4 * q + 3] = w.w;
                    }
#pragma unroll
                    for (int hi = 0; hi < 2; ++hi) {
                        const uint8_t *ks = blk + LY::k_scale(0, 0) + (gid + 8 * hi) * NG * 2;
                        if constexpr (NG == 4) {
                            const uint2 w = *reinterpret_cast<const uint2 *>(ks);
                            kss[b][2 * hi] = w.x;
                            kss[b][2 * hi + 1] = w.y;
                        } else {
                            kss[b][hi] = *reinterpret_cast<const uint32_t *>(ks);
                        }
                    }
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        sc[b][nb][0] = sc[b][nb][1] = sc[b][nb][2] = sc[b][nb][3] = 0.f;
                }
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    uint4 q[NB];
                    float2 bias[NB];
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        q[nb] = *reinterpret_cast<const uint4 *>(
                            smem + PL::kQ + (8 * nb + gid) * PL::kQRow + g * 64 + tig * 16);
                        bias[nb] = *reinterpret_cast<const float2 *>(
                            smem + PL::kBias + (g * 16 + 8 * nb + 2 * tig) * 4);
                    }
#pragma unroll
                    for (int b = 0; b < NS; ++b) {
                        const uint32_t w0 = kw[b][g], w1 = kw[b][NG + g];
                        const uint32_t s0 = kss[b][g / 2], s1 = kss[b][NG / 2 + g / 2];
                        const float f0 = (g & 1) ? bf16_hi(s0) : bf16_lo(s0);
                        const float f1 = (g & 1) ? bf16_hi(s1) : bf16_lo(s1);
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) {
                            float t[4];
                            mma_from(t, codes_at(w0, 0), codes_at(w1, 0), codes_at(w0, 1),
                                     codes_at(w1, 1), q[nb].x, q[nb].y, bias[nb].x, bias[nb].y,
                                     bias[nb].x, bias[nb].y);
                            mma_from(t, codes_at(w0, 2), codes_at(w1, 2), codes_at(w0, 3),
                                     codes_at(w1, 3), q[nb].z, q[nb].w, t[0], t[1], t[2], t[3]);
                            sc[b][nb][0] = fmaf(t[0], f0, sc[b][nb][0]);
                            sc[b][nb][1] = fmaf(t[1], f0, sc[b][nb][1]);
                            sc[b][nb][2] = fmaf(t[2], f1, sc[b][nb][2]);
                            sc[b][nb][3] = fmaf(t[3], f1, sc[b][nb][3]);
                        }
                    }
                }
                if (edge) {
                    // Positions outside [vis0, vis1) hold anything, NaN scales among it.
#pragma unroll
                    for (int b = 0; b < NS; ++b)
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const int r = 16 * b + gid + 8 * (c >> 1);
                            if (r < vis0 || r >= vis1) {
#pragma unroll
                                for (int nb = 0; nb < NB; ++nb)
                                    sc[b][nb][c] = NEG_INF;
                            }
                        }
                }
                // ---- online softmax (base 2), the reference maximum raised rarely ----
                uint32_t pb[NS][NB][2];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    float mx[2] = {NEG_INF, NEG_INF};
#pragma unroll
                    for (int b = 0; b < NS; ++b) {
                        mx[0] = fmaxf(mx[0], fmaxf(sc[b][nb][0], sc[b][nb][2]));
                        mx[1] = fmaxf(mx[1], fmaxf(sc[b][nb][1], sc[b][nb][3]));
                    }
                    const bool raise = mx[0] * p.scale_log2 > m_run[nb][0] + kQ4LazyMax ||
                                       mx[1] * p.scale_log2 > m_run[nb][1] + kQ4LazyMax;
                    if (__any_sync(0xffffffffu, raise)) {
                        float alpha[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 4));
                            mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 8));
                            mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 16));
                            const float m_new = fmaxf(m_run[nb][i], mx[i] * p.scale_log2);
                            alpha[i] = m_new == NEG_INF ? 1.f : fast_exp2(m_run[nb][i] - m_new);
                            m_run[nb][i] = m_new;
                        }
#pragma unroll
                        for (int n = 0; n < 2 * NG; ++n) {
                            o[nb][n][0] *= alpha[0];
                            o[nb][n][1] *= alpha[1];
                            o[nb][n][2] *= alpha[0];
                            o[nb][n][3] *= alpha[1];
                        }
                        la[nb][0] *= alpha[0];
                        la[nb][1] *= alpha[1];
                    }
                    const float m0 = m_run[nb][0] == NEG_INF ? 0.f : m_run[nb][0];
                    const float m1 = m_run[nb][1] == NEG_INF ? 0.f : m_run[nb][1];
#pragma unroll
                    for (int b = 0; b < NS; ++b) {
                        const float p0 = fast_exp2(fmaf(sc[b][nb][0], p.scale_log2, -m0));
                        const float p1 = fast_exp2(fmaf(sc[b][nb][1], p.scale_log2, -m1));
                        const float p2 = fast_exp2(fmaf(sc[b][nb][2], p.scale_log2, -m0));
                        const float p3 = fast_exp2(fmaf(sc[b][nb][3], p.scale_log2, -m1));
                        pb[b][nb][0] = movmatrix_trans(pack_bf16x2(p0, p1));
                        pb[b][nb][1] = movmatrix_trans(pack_bf16x2(p2, p3));
                        mma_from(la[nb], kOnes2, kOnes2, kOnes2, kOnes2, pb[b][nb][0], pb[b][nb][1],
                                 la[nb][0], la[nb][1], la[nb][2], la[nb][3]);
                    }
                }
                // ---- O += V^T (s P)^T ----
                uint32_t vw[NS][2 * NG], vs[NS][2 * NG];   // [th][group]
#pragma unroll
                for (int b = 0; b < NS; ++b) {
                    const uint8_t *blk = st + b * LY::kBytes;
#pragma unroll
                    for (int q = 0; q < 2 * NG / 4; ++q) {
                        const uint4 w =
                            *reinterpret_cast<const uint4 *>(blk + LY::kV + q * 512 + lane * 16);
                        vw[b][4 * q] = w.x;
                        vw[b][4 * q + 1] = w.y;
                        vw[b][4 * q + 2] = w.z;
                        vw[b][4 * q + 3] = w.w;
                        const uint4 f = *reinterpret_cast<const uint4 *>(
                            blk + LY::kVs + tig * NG * 8 + q * 16);
                        vs[b][4 * q] = f.x;
                        vs[b][4 * q + 1] = f.y;
                        vs[b][4 * q + 2] = f.z;
                        vs[b][4 * q + 3] = f.w;
                    }
                    if (edge) {
#pragma unroll
                        for (int th = 0; th < 2; ++th) {
                            const int r = 16 * b + 8 * th + 2 * tig;
                            const uint32_t keep = (r >= vis0 && r < vis1 ? 0x0000ffffu : 0u) |
                                                  (r + 1 >= vis0 && r + 1 < vis1 ? 0xffff0000u : 0u);
#pragma unroll
                            for (int g = 0; g < NG; ++g)
                                vs[b][th * NG + g] &= keep;
                        }
                    }
                }
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    uint32_t pv[NS][NB][2];
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        float t0[4] = {0.f, 0.f, 0.f, 0.f}, t1[4];
#pragma unroll
                        for (int b = 0; b < NS; ++b) {
                            pv[b][nb][0] = hmul2_bf16(pb[b][nb][0], vs[b][g]);
                            pv[b][nb][1] = hmul2_bf16(pb[b][nb][1], vs[b][NG + g]);
                            mma_from(t0, kMinus136, kMinus136, kMinus136, kMinus136, pv[b][nb][0],
                                     pv[b][nb][1], t0[0], t0[1], t0[2], t0[3]);
                        }
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            t1[c] = t0[c];
#pragma unroll
                        for (int b = 0; b < NS; ++b) {
                            const uint32_t w0 = vw[b][g], w1 = vw[b][NG + g];
                            mma_from(t0, codes_at(w0, 0), codes_at(w0, 1), codes_at(w1, 0),
                                     codes_at(w1, 1), pv[b][nb][0], pv[b][nb][1], t0[0], t0[1], t0[2],
                                     t0[3]);
                            mma_from(t1, codes_at(w0, 2), codes_at(w0, 3), codes_at(w1, 2),
                                     codes_at(w1, 3), pv[b][nb][0], pv[b][nb][1], t1[0], t1[1], t1[2],
                                     t1[3]);
                        }
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            o[nb][2 * g][c] += t0[c];
                            o[nb][2 * g + 1][c] += t1[c];
                        }
                    }
                }
            }
            __syncwarp();
            fetch();   // into the stage just read
        }

        // ---- end of the piece: the warps' sums are merged, 8 heads at a time ----
        float *raw = reinterpret_cast<float *>(smem + PL::kRaw);          // [kWarps][8][kRow]
        float *st_m = reinterpret_cast<float *>(smem + PL::kStat);        // [8 NB][kWarps]
        float *st_l = st_m + 8 * NB * NW;
        const int G = p.G, seg = cs.beta * p.g + cs.j;
        const bool whole = piece == cs.first && piece_end == seg_end;
        const size_t rec = static_cast<size_t>(seg) + cta;
        __nv_bfloat16 *ob =
            p.out + (static_cast<size_t>(cs.beta) * p.h + static_cast<size_t>(cs.j) * G) * D;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            if (nb > 0 && G <= 8 * nb)
                break;
            if (nb > 0)
                __syncthreads();   // the sums of the heads before have been read
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float *dst = raw + (warp * 8 + 2 * tig + i) * PL::kRow + gid * 4;
#pragma unroll
                for (int g = 0; g < NG; ++g)
                    *reinterpret_cast<float4 *>(dst + g * 32) =
                        make_float4(o[nb][2 * g][i], o[nb][2 * g][2 + i], o[nb][2 * g + 1][i],
                                    o[nb][2 * g + 1][2 + i]);
                if (gid == 0) {
                    st_m[(8 * nb + 2 * tig + i) * NW + warp] = m_run[nb][i];
                    st_l[(8 * nb + 2 * tig + i) * NW + warp] = la[nb][i];
                }
            }
            __syncthreads();
            const int rows = min(G - 8 * nb, 8);
            for (int i = 4 * tid; i < rows * D; i += 4 * PL::kThreads) {
                const int row = i / D, e = i - row * D;
                float ms = NEG_INF;   // finite below: the piece holds a visible position
#pragma unroll
                for (int w = 0; w < NW; ++w)
                    ms = fmaxf(ms, st_m[(8 * nb + row) * NW + w]);
                float ls = 0.f;
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    const float f = fast_exp2(st_m[(8 * nb + row) * NW + w] - ms);
                    ls = fmaf(st_l[(8 * nb + row) * NW + w], f, ls);
                    const float4 x =
                        *reinterpret_cast<const float4 *>(raw + (w * 8 + row) * PL::kRow + e);
                    v.x = fmaf(f, x.x, v.x);
                    v.y = fmaf(f, x.y, v.y);
                    v.z = fmaf(f, x.z, v.z);
                    v.w = fmaf(f, x.w, v.w);
                }
                const float inv = fast_rcp(ls);
                v.x *= inv;
                v.y *= inv;
                v.z *= inv;
                v.w *= inv;
                const int at = 8 * nb * D + i;
                if (whole) {
                    *reinterpret_cast<uint2 *>(ob + at) =
                        make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
                } else {
                    *reinterpret_cast<float4 *>(p.part_o + rec * G * D + at) = v;
                    if (e == 0)
                        p.part_lse[rec * G + 8 * nb + row] = ms + fast_log2(ls);
                }
            }
        }
        if (!last)
            store_q(q_next);   // every warp has passed this piece's last use of the queries
        if (!whole && !p.deferred_merge) {
            // The CTA that finishes a segment last merges its records, in their order.
            const int c0 = cta_of_tile(cs.first, N, P), c1 = cta_of_tile(seg_end - 1, N, P);
            __syncthreads();
            if (tid == 0)
                flags[1] = atomic_add_acq_rel_gpu(&p.counters[seg], 1u) ==
                           static_cast<unsigned>(c1 - c0);
            __syncthreads();
            if (flags[1]) {
                const int np = c1 - c0 + 1;
                const size_t rec0 = static_cast<size_t>(seg) + c0;
                for (int i = 4 * tid; i < G * D; i += 4 * PL::kThreads) {
                    const int row = i / D;
                    float l[kInlineMergeMaxPieces];
                    float4 x[kInlineMergeMaxPieces];
                    float mx = NEG_INF;
#pragma unroll
                    for (int k = 0; k < kInlineMergeMaxPieces; ++k) {
                        l[k] = NEG_INF;
                        x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (k < np) {
                            l[k] = __ldcg(&p.part_lse[(rec0 + k) * G + row]);
                            x[k] = __ldcg(reinterpret_cast<const float4 *>(
                                p.part_o + (rec0 + k) * G * D + i));
                        }
                        mx = fmaxf(mx, l[k]);
                    }
                    float tot = 0.f;
                    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int k = 0; k < kInlineMergeMaxPieces; ++k) {
                        const float f = fast_exp2(l[k] - mx);   // 0 past the records
                        tot += f;
                        a.x = fmaf(f, x[k].x, a.x);
                        a.y = fmaf(f, x[k].y, a.y);
                        a.z = fmaf(f, x[k].z, a.z);
                        a.w = fmaf(f, x[k].w, a.w);
                    }
                    const float inv = fast_rcp(tot);
                    *reinterpret_cast<uint2 *>(ob + i) =
                        make_uint2(pack_bf16x2(a.x * inv, a.y * inv), pack_bf16x2(a.z * inv, a.w * inv));
                }
                if (tid == 0)
                    p.counters[seg] = 0u;
            }
        }
        __syncthreads();   // the next piece's queries are in place; sums and flags may be rewritten
        piece = piece_end;
        cs = ns;
    }
    // No copy may still be in flight when the CTA exits (after an expired wait).
    if (lane == 0 && flags[0]) {
        for (int k = f_it > R ? f_it - R : 0; k < f_it; ++k)
            if (!mbar_wait(bar_full + 8 * (k % R), (k / R) & 1))
                atomicOr(p.err, kErrDrain);
    }
}

template <int D, int NB>
struct Launch {
    static const void *fn() { return reinterpret_cast<const void *>(&q4_decode_kernel<D, NB>); }
};

const void *decode_fn(int d, int group, int *threads, size_t *smem)
{
    if (d == 64) {
        *threads = Q4Plan<64, 1>::kThreads;
        *smem = group <= 8 ? Q4Plan<64, 1>::kBytes : Q4Plan<64, 2>::kBytes;
        return group <= 8 ? Launch<64, 1>::fn() : Launch<64, 2>::fn();
    }
    *threads = Q4Plan<128, 1>::kThreads;
    *smem = group <= 8 ? Q4Plan<128, 1>::kBytes : Q4Plan<128, 2>::kBytes;
    return group <= 8 ? Launch<128, 1>::fn() : Launch<128, 2>::fn();
}

}  // namespace

cudaError_t prepare_q4_decode(int d, int group, int *ctas_per_sm)
{
    int threads;
    size_t smem;
    const void *fn = decode_fn(d, group, &threads, &smem);
    cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         static_cast<int>(smem));
    if (e != cudaSuccess)
        return e;
    return cudaOccupancyMaxActiveBlocksPerMultiprocessor(ctas_per_sm, fn, threads, smem);
}

cudaError_t launch_q4_decode(int d, int grid, const Q4DecodeParams &p, cudaStream_t stream)
{
    int threads;
    size_t smem;
    const void *fn = decode_fn(d, p.G, &threads, &smem);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    void *args[] = {const_cast<Q4DecodeParams *>(&p)};
    return cudaLaunchKernelExC(&cfg, fn, args);
}

}  // namespace mlkv
