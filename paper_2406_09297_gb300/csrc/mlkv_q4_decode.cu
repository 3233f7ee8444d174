// Single-token decode attention over the 4-bit KV cache (layout and values: mlkv_q4.h), with an
// optional sliding window and sinks (MLKV, arXiv 2406.09297, Sec. 3; attention of Eqs. 2-3).
//
//   out = sum_t p_t v_t / sum_t p_t,  p_t = 2^(log2(e) q.k_t / sqrt(D) - m)
//
// What bounds it: at 0.5625 bytes a channel HBM delivers ~42 channels per SM and clock, so unpacking is
// the work to be saved.  K and V are never widened: one shift and one AND turn a quarter of a word of
// 8 codes into a register of the A operand, fp16 with the code's magnitude in units of 2^-16 (mlkv_q4.h).
//   S = K Q^T, 16 positions by 8 heads a group of 32 channels: exact codes, queries as fp16 scaled by a
//       power of two per head to at most 2^15 (bf16's 8 bits fit; below 2^-29 of the head's largest
//       magnitude bits are lost); fp32 sums, times the group's scale in fp32.
//   O = V^T P^T, 16 channels by 8 heads.  The group's scale goes into P: P' = fp16(fp16(p) s / f), f a
//       power of two that bounds the scales the warp has met (raised with a rescaled O, like the
//       running maximum), so that fp16's range holds whatever the values' magnitude.
// (Tried before.  Codes as bf16 128 + c, the surplus cancelled in the accumulators, P in bf16: as fast,
// outputs 0.0024 to 0.0029 from the 64-bit ones instead of 0.0017.  K in e4m3: mma.sync takes 8-bit
// operands apart again, 385 instructions per 16 positions of 128 channels and 8 heads.)
//
// Work split as in decode_kernel: the tiles of all (sequence, KV head) segments end to end, an equal run
// of them for each persistent CTA; a CTA's warps take its tiles in turn, each through a ring of its own
// (one bulk copy a tile: a block's codes and scales lie together), so nothing but the ends of
// segments makes warps wait for one another.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
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
    // The piece's queries as fp16, a lane's 8 channels of a group 16 bytes, the odd heads' halves of 128
    // bytes swapped so that a quarter warp's loads fall in distinct banks; and what a head's products
    // are to be multiplied with.
    static constexpr int kQRow = 2 * D;
    static constexpr int kQ = kStat + 2 * 8 * NB * kWarps * 4;
    static constexpr int kMul = kQ + 8 * NB * kQRow;
    static constexpr int kVs = kMul + 8 * NB * 4;               // [kWarps][64] V scales, fp16 pairs
    static constexpr int kFlags = kVs + kWarps * 256;
    static constexpr int kBars = kFlags + 16;
    static constexpr int kBytes = kBars + kWarps * kStages * 8;
    static_assert(kSub * 8 * LY::kGroups == 64, "two words of V scales a lane");
    static_assert(kMinBlocks * (kBytes + 1024) <= 228 * 1024, "shared memory of the resident CTAs");
    static_assert(kTileBytes % 128 == 0 && kRaw % 16 == 0 && kQ % 16 == 0 && kVs % 16 == 0 &&
                      kBars % 8 == 0, "");
    __device__ static constexpr int q_at(int head, int group, int tig)
    {
        return kQ + head * kQRow + (((group * 4 + tig) ^ ((head & 1) * 4)) * 16);
    }
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

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                        uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 "
        "{%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

__device__ __forceinline__ uint32_t hmul2_f16(uint32_t a, uint32_t b)
{
    const __half2 x = *reinterpret_cast<const __half2 *>(&a);
    const __half2 y = *reinterpret_cast<const __half2 *>(&b);
    const __half2 z = __hmul2(x, y);
    return *reinterpret_cast<const uint32_t *>(&z);
}

// Reference maxima move when a score exceeds them by more than this (log2 units): weights stay <= 2^8.
constexpr float kQ4LazyMax = 8.f;

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
    // Queries of a segment: 16 bytes (8 channels) a thread, a head's threads neighbours in a warp.
    constexpr int kOct = D / 8;
    constexpr int kQThreads = 8 * NB * kOct;
    static_assert(kQThreads <= PL::kThreads, "one load a thread");
    auto load_q = [&](const Segment &s) {
        const int head = tid / kOct;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (tid < kQThreads && head < p.G)
            v = *reinterpret_cast<const uint4 *>(
                p.Q + (static_cast<size_t>(s.beta) * p.h + static_cast<size_t>(s.j) * p.G) * D +
                tid * 8);
        return v;
    };
    auto store_q = [&](const uint4 &v) {
        if (tid >= kQThreads)   // whole warps
            return;
        const int head = tid / kOct, oct = tid % kOct;
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        // a row with a NaN or an infinity becomes NaN
        auto bad_row = [](float m) { return !(m < __int_as_float(0x7f800000)); };
        float x[8], mx = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = (i & 1) ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
            mx = fmaxf(mx, bad_row(fabsf(x[i])) ? __int_as_float(0x7f800000) : fabsf(x[i]));
        }
#pragma unroll
        for (int m = 1; m < kOct; m <<= 1)
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, m));
        // 2^e, the largest with mx 2^e < 2^15 (within limits that keep every factor finite)
        const int e = max(-100, min(100, 14 - (static_cast<int>(__float_as_uint(mx) >> 23) - 127)));
        const float up = __int_as_float((127 + e) << 23), down = __int_as_float((127 - e) << 23);
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            y[i] = bad_row(mx) ? 0x7fff7fffu : pack_f16x2(x[2 * i] * up, x[2 * i + 1] * up);
        *reinterpret_cast<uint4 *>(smem + PL::q_at(head, oct >> 2, oct & 3)) =
            make_uint4(y[0], y[1], y[2], y[3]);
        if (oct == 0)
            reinterpret_cast<float *>(smem + PL::kMul)[head] = p.scale_log2 * kQ4Unit * down;
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
        // A thread's statistics are those of heads 2 tig and 2 tig + 1 (la: over its own positions);
        // O is in units of 2^-16 times the scales' bound.
        float o[NB][2 * NG][4];
        float la[NB][2], m_run[NB][2], mul[NB][2];
        float bound = 0x1p-100f, inv_bound = 0x1p100f;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int n = 0; n < 2 * NG; ++n)
                o[nb][n][0] = o[nb][n][1] = o[nb][n][2] = o[nb][n][3] = 0.f;
            la[nb][0] = la[nb][1] = 0.f;
            m_run[nb][0] = m_run[nb][1] = NEG_INF;
            const float2 f =
                *reinterpret_cast<const float2 *>(smem + PL::kMul + (8 * nb + 2 * tig) * 4);
            mul[nb][0] = f.x;
            mul[nb][1] = f.y;
        }
        uint32_t *vscale = reinterpret_cast<uint32_t *>(smem + PL::kVs) + warp * 64;
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
                // ---- the scales of V as fp16, over their bound: two pairs a lane ----
                float2 vf[2];
                float top = 0.f;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int k = lane + 32 * i, blk = k / (8 * NG), at = k % (8 * NG);
                    const uint32_t w = *reinterpret_cast<const uint32_t *>(st + blk * LY::kBytes +
                                                                           LY::kVs + at * 4);
                    vf[i] = make_float2(bf16_lo(w), bf16_hi(w));
                    if (edge) {
                        // positions outside [vis0, vis1) hold anything, NaN scales among it
                        const int r = 16 * blk + 8 * (at / NG & 1) + 2 * (at / (2 * NG));
                        if (r < vis0 || r >= vis1)
                            vf[i].x = 0.f;
                        if (r + 1 < vis0 || r + 1 >= vis1)
                            vf[i].y = 0.f;
                    }
                    top = fmaxf(top, fmaxf(vf[i].x, vf[i].y));
                }
                if (__any_sync(0xffffffffu, top > bound)) {
#pragma unroll
                    for (int m = 1; m < 32; m <<= 1)
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
                    // the power of two above it (scales are below 2^126)
                    const uint32_t eb = (__float_as_uint(top) >> 23) + 1;
                    const float down = bound * __uint_as_float((254u - eb) << 23);
                    bound = __uint_as_float(eb << 23);
                    inv_bound = __uint_as_float((254u - eb) << 23);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int n = 0; n < 2 * NG; ++n)
#pragma unroll
                            for (int c = 0; c < 4; ++c)
                                o[nb][n][c] *= down;
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    vscale[lane + 32 * i] = pack_f16x2(vf[i].x * inv_bound, vf[i].y * inv_bound);
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
                }
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    uint4 q[NB];
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        q[nb] =
                            *reinterpret_cast<const uint4 *>(smem + PL::q_at(8 * nb + gid, g, tig));
#pragma unroll
                    for (int b = 0; b < NS; ++b) {
                        const uint32_t w0 = kw[b][g], w1 = kw[b][NG + g];
                        const uint32_t a[8] = {q4_pair(w0, 0), q4_pair(w1, 0), q4_pair(w0, 1), q4_pair(w1, 1),
                                               q4_pair(w0, 2), q4_pair(w1, 2), q4_pair(w0, 3), q4_pair(w1, 3)};
                        const uint32_t s0 = kss[b][g / 2], s1 = kss[b][NG / 2 + g / 2];
                        const float f0 = (g & 1) ? bf16_hi(s0) : bf16_lo(s0);
                        const float f1 = (g & 1) ? bf16_hi(s1) : bf16_lo(s1);
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) {
                            float t[4] = {0.f, 0.f, 0.f, 0.f};
                            mma_f16(t, a[0], a[1], a[2], a[3], q[nb].x, q[nb].y);
                            mma_f16(t, a[4], a[5], a[6], a[7], q[nb].z, q[nb].w);
                            sc[b][nb][0] = g == 0 ? t[0] * f0 : fmaf(t[0], f0, sc[b][nb][0]);
                            sc[b][nb][1] = g == 0 ? t[1] * f0 : fmaf(t[1], f0, sc[b][nb][1]);
                            sc[b][nb][2] = g == 0 ? t[2] * f1 : fmaf(t[2], f1, sc[b][nb][2]);
                            sc[b][nb][3] = g == 0 ? t[3] * f1 : fmaf(t[3], f1, sc[b][nb][3]);
                        }
                    }
                }
                if (edge) {
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
                    const bool raise = mx[0] * mul[nb][0] > m_run[nb][0] + kQ4LazyMax ||
                                       mx[1] * mul[nb][1] > m_run[nb][1] + kQ4LazyMax;
                    if (__any_sync(0xffffffffu, raise)) {
                        float alpha[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 4));
                            mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 8));
                            mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 16));
                            const float m_new = fmaxf(m_run[nb][i], mx[i] * mul[nb][i]);
                            alpha[i] = m_new == NEG_INF ? 1.f : fast_exp2(m_run[nb][i] - m_new);
                            m_run[nb][i] = m_new;
                            la[nb][i] *= alpha[i];
                        }
#pragma unroll
                        for (int n = 0; n < 2 * NG; ++n) {
                            o[nb][n][0] *= alpha[0];
                            o[nb][n][1] *= alpha[1];
                            o[nb][n][2] *= alpha[0];
                            o[nb][n][3] *= alpha[1];
                        }
                    }
                    const float m0 = m_run[nb][0] == NEG_INF ? 0.f : m_run[nb][0];
                    const float m1 = m_run[nb][1] == NEG_INF ? 0.f : m_run[nb][1];
#pragma unroll
                    for (int b = 0; b < NS; ++b) {
                        const float p0 = fast_exp2(fmaf(sc[b][nb][0], mul[nb][0], -m0));
                        const float p1 = fast_exp2(fmaf(sc[b][nb][1], mul[nb][1], -m1));
                        const float p2 = fast_exp2(fmaf(sc[b][nb][2], mul[nb][0], -m0));
                        const float p3 = fast_exp2(fmaf(sc[b][nb][3], mul[nb][1], -m1));
                        la[nb][0] += p0 + p2;
                        la[nb][1] += p1 + p3;
                        pb[b][nb][0] = movmatrix_trans(pack_f16x2(p0, p1));
                        pb[b][nb][1] = movmatrix_trans(pack_f16x2(p2, p3));
                    }
                }
                __syncwarp();   // the scales of V are in place
                // ---- O += V^T (s P)^T ----
#pragma unroll
                for (int b = 0; b < NS; ++b) {
                    const uint8_t *blk = st + b * LY::kBytes;
                    uint32_t vw[2 * NG], vs[2 * NG];   // [th][group]
#pragma unroll
                    for (int q = 0; q < 2 * NG / 4; ++q) {
                        const uint4 w =
                            *reinterpret_cast<const uint4 *>(blk + LY::kV + q * 512 + lane * 16);
                        vw[4 * q] = w.x;
                        vw[4 * q + 1] = w.y;
                        vw[4 * q + 2] = w.z;
                        vw[4 * q + 3] = w.w;
                        const uint4 f = *reinterpret_cast<const uint4 *>(
                            vscale + b * 8 * NG + tig * 2 * NG + q * 4);
                        vs[4 * q] = f.x;
                        vs[4 * q + 1] = f.y;
                        vs[4 * q + 2] = f.z;
                        vs[4 * q + 3] = f.w;
                    }
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        const uint32_t w0 = vw[g], w1 = vw[NG + g];
                        const uint32_t a[8] = {q4_pair(w0, 0), q4_pair(w0, 1), q4_pair(w1, 0),
                                               q4_pair(w1, 1), q4_pair(w0, 2), q4_pair(w0, 3),
                                               q4_pair(w1, 2), q4_pair(w1, 3)};
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) {
                            const uint32_t b0 = hmul2_f16(pb[b][nb][0], vs[g]);
                            const uint32_t b1 = hmul2_f16(pb[b][nb][1], vs[NG + g]);
                            mma_f16(o[nb][2 * g], a[0], a[1], a[2], a[3], b0, b1);
                            mma_f16(o[nb][2 * g + 1], a[4], a[5], a[6], a[7], b0, b1);
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
        // out of the units of the codes and of the scales' bound (whose product may pass fp32's range)
        auto whole_units = [&](float x) { return x * kQ4Unit * bound; };
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                la[nb][i] += __shfl_xor_sync(0xffffffffu, la[nb][i], 4);
                la[nb][i] += __shfl_xor_sync(0xffffffffu, la[nb][i], 8);
                la[nb][i] += __shfl_xor_sync(0xffffffffu, la[nb][i], 16);
            }
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
                        make_float4(whole_units(o[nb][2 * g][i]), whole_units(o[nb][2 * g][2 + i]),
                                    whole_units(o[nb][2 * g + 1][i]),
                                    whole_units(o[nb][2 * g + 1][2 + i]));
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
