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
//   O = V^T P^T, 16 channels by 8 heads.  The group's scale goes into P: P' = fp16(p s u), p s in fp32, u a
//       power of two of the head and group that follows the largest product p s the warp has met (with a
//       rescaled O, like the running maximum, and rarely: a bound on the scales tells when it may have to).  A
//       scale thus counts with its weight, and a group by itself: each product is off by 2^-11 of itself, and
//       below 2^-16 of the largest by up to 2^-27 of that.  (With fp16(p) times fp16(s / f), one f for all
//       groups and positions, 6 to 10% faster, a large value of no weight or a sink of small value drove the
//       others below fp16's range: errors of percents to 100%.)
// Measured on GB300, one layer, 8 KV heads of 128 with 4 query heads each, us (TB/s of 6.8): 128 sequences
// of 4096 positions 109.5 (5.5), 64 61.4 (4.9), 32 33.1 (4.6), 64 uneven ones of up to 8192 60.0 (4.7).
// Twice the sequences cost 48.1 us more for 44.4 us more of bytes; beside that there are ~3 us of start and, at
// the end, warps that finish up to 12 us apart and then merge for 3 to 5 us.  One sequence of 131072, 12 heads
// of 64 over one KV head: 11.7, two launches' latencies.
// (Tried before.  Codes as bf16 128 + c, the surplus cancelled in the accumulators, P in bf16: outputs 0.0024 to
// 0.0029 from the 64-bit ones instead of 0.0017.  K in e4m3: mma.sync takes 8-bit
// operands apart again, 385 instructions per 16 positions of 128 channels and 8 heads.)
//
// Work split.  The tiles of all (sequence, KV head) segments end to end, an equal run of them for each
// worker, the part of a segment in one run a piece.  Every warp has a ring of its own (one bulk copy a tile: a
// block's codes and scales lie together).  With many tiles a worker is a warp, which meets no other until
// it stores its pieces: no barrier, and a piece of a few tiles costs its warp a round trip or two while
// the others stream.  With few, it is a CTA, whose warps take its tiles in turn and merge their sums at its
// end; segments are filled up with empty tiles so that a run holds tiles of one of them.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "mlkv_q4.h"

#include "mlkv_device.cuh"

namespace mlkv {
namespace {

// kWarpRuns: every warp has a run of tiles, and the queries of its segment, of its own; else a CTA's warps
// share both.
template <int D, int NB, bool kWarpRuns>
struct Q4Plan {
    using LY = Q4Layout<D>;
    static constexpr int kWarps = q4_warps(D, 8 * NB);
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kT = q4_tile_tokens(D);
    static constexpr int kSub = kT / kQ4Block;                  // blocks of a tile
    static constexpr int kStages = 2;
    static constexpr int kTileBytes = kSub * LY::kBytes;
    static constexpr int kMinBlocks = 2;
    static constexpr int kRing = 0;                             // [kWarps][kStages]
    // The queries as fp16, a lane's 8 channels of a group 16 bytes, the odd heads' halves of 128 bytes
    // swapped so that a quarter warp's loads fall in distinct banks; and what a head's products are to
    // be multiplied with.
    static constexpr int kQSets = kWarpRuns ? kWarps : 1;
    static constexpr int kQRow = 2 * D;
    static constexpr int kQ = kRing + kWarps * kStages * kTileBytes;
    static constexpr int kQSet = 8 * NB * kQRow;
    static constexpr int kMul = kQ + kQSets * kQSet;
    static constexpr int kBars = kMul + kQSets * 8 * NB * 4;
    static constexpr int kFlags = kBars + kWarps * kStages * 8;
    // Shared runs: a piece's sums of 8 heads from every warp, rows padded so that the fragments' 16-byte
    // stores fall in distinct banks, and m, l [8 NB heads][kWarps].
    static constexpr int kRow = D + 4;
    static constexpr int kRaw = kFlags + 16;
    static constexpr int kStat = kRaw + (kWarpRuns ? 0 : kWarps * 8 * kRow * 4);
    static constexpr int kBytes = kStat + (kWarpRuns ? 0 : 2 * 8 * NB * kWarps * 4);
    static_assert(kMinBlocks * (kBytes + 1024) <= 228 * 1024, "shared memory of the resident CTAs");
    static_assert(kTileBytes % 128 == 0 && kQ % 16 == 0 && kBars % 8 == 0 && kRaw % 16 == 0, "");
    __device__ static constexpr int q_at(int head, int group, int tig)
    {
        return kQ + head * kQRow + (((group * 4 + tig) ^ ((head & 1) * 4)) * 16);
    }
};

// A (sequence, KV head) segment as the walk sees it.
struct Segment {
    int beta, j, L;
    int first, nt;        // its first tile in the flattened list, its tiles with the empty ones behind
    VisibleTiles v;
};

template <int T>
__device__ __forceinline__ void load_segment(const Q4DecodeParams &p, Segment &s)
{
    s.L = p.uniform_len > 0 ? p.uniform_len : p.seq_len[s.beta];
    s.v = visible_tiles(s.L, p.window, p.sinks, T, kQ4Block);
    s.nt = p.round_tiles > 0 ? (s.v.nt + p.round_tiles - 1) / p.round_tiles * p.round_tiles
                             : s.v.nt + p.empty_tiles;
}

template <int T>
__device__ __forceinline__ Segment segment_of_tile(const Q4DecodeParams &p, int tile)
{
    Segment s;
    if (p.uniform_len > 0) {
        s.beta = 0;
        load_segment<T>(p, s);
        const int seg = tile / s.nt;
        s.beta = seg / p.g;
        s.j = seg - s.beta * p.g;
        s.first = seg * s.nt;
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
    s.j = (tile - p.tile_start[lo]) / s.nt;
    s.first = p.tile_start[lo] + s.j * s.nt;
    return s;
}

template <int T>
__device__ __forceinline__ void next_segment(const Q4DecodeParams &p, Segment &s)
{
    s.first += s.nt;
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

// The first product of a sum.
__device__ __forceinline__ void mma_f16_zero(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                             uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 "
        "{%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// 1 / x, x a power of two in [2^-126, 2^126].
__device__ __forceinline__ float reciprocal2(float x)
{
    return __uint_as_float((254u << 23) - __float_as_uint(x));
}

// A head's reference lies this much (log2 units) above its largest score when it is set, and moves when a
// score exceeds it: weights are at most 1.
constexpr float kQ4LazyMax = 4.f;
// A power of two of a head and group brings their largest product of weight and scale to
// [2^kQ4ProductTop, 2^(kQ4ProductTop + 1)) when it is set, and moves when one reaches 2^15.  As weights are
// at most 1, scales below 2^15 over the largest power of two need no look at the products.  (128 sequences of
// 4096 that begin with a sink of 12 nats and values 0.02 of the others', us: 2^7 and 3 log2 units 148, 2^3 and
// 5 125, these 110, as without the sink.)
constexpr uint32_t kQ4ProductTop = 2;
constexpr float kQ4ProductMost = 32768.f;
constexpr uint32_t kQ4UpNone = 0x7e807e80u;   // bf16 pair of 2^126: nothing met yet, and the largest power

template <int D, int NB, bool kWarpRuns>
__global__ void __launch_bounds__(Q4Plan<D, NB, kWarpRuns>::kThreads,
                                  Q4Plan<D, NB, kWarpRuns>::kMinBlocks)
    q4_decode_kernel(const __grid_constant__ Q4DecodeParams p)
{
    using PL = Q4Plan<D, NB, kWarpRuns>;
    using LY = Q4Layout<D>;
    constexpr int NW = PL::kWarps, T = PL::kT, NS = PL::kSub, NG = LY::kGroups, R = PL::kStages;
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t sbase = smem_addr(smem);
    volatile int *flags = reinterpret_cast<volatile int *>(smem + PL::kFlags);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int gid = lane >> 2, tig = lane & 3;
    // run `run` of P: tiles [tile_lo, tile_hi), of which this warp takes every kStep-th
    const int P = gridDim.x * (kWarpRuns ? NW : 1), N = p.num_tiles;
    const int run = kWarpRuns ? blockIdx.x * NW + warp : blockIdx.x;
    const int tile_lo = static_cast<int>(static_cast<long long>(run) * N / P);
    const int tile_hi = static_cast<int>(static_cast<long long>(run + 1) * N / P);
    constexpr int kStep = kWarpRuns ? 1 : NW;
    const int tile_first = tile_lo + (kWarpRuns ? 0 : warp);
    const uint32_t ring = sbase + PL::kRing + warp * R * PL::kTileBytes;
    const uint32_t bar_full = sbase + PL::kBars + warp * R * 8;
    // this warp's queries and their factors
    const uint8_t *q_set = smem + (kWarpRuns ? warp * PL::kQSet : 0);
    float *q_mul = reinterpret_cast<float *>(smem + PL::kMul) + (kWarpRuns ? warp * 8 * NB : 0);
    bool expired = false;   // a wait gave up
    const float NEG_INF = -__int_as_float(0x7f800000);
    if (lane == 0) {
        for (int s = 0; s < R; ++s)
            mbar_init(bar_full + 8 * s, 1);
        fence_barrier_init();
    }
    __syncwarp();

    // Lane 0 sends the copies of the warp's tiles R ahead; f_run of them follow one another at f_src.
    Segment fs = segment_of_tile<T>(p, tile_lo < N ? tile_lo : N - 1);
    // where the tiles to read end (a CTA's run lies in one segment, filled up with empty tiles)
    const int tile_end = kWarpRuns ? tile_hi : min(tile_hi, fs.first + fs.v.nt);
    int f_tile = tile_first, f_it = 0, f_run = 0;
    const uint8_t *f_src = nullptr;
    auto send = [&](uint32_t bytes) {
        const int s = f_it % R;
        mbar_arrive_expect_tx(bar_full + 8 * s, bytes);
        bulk_load(ring + s * PL::kTileBytes, f_src, bytes, bar_full + 8 * s);
        f_tile += kStep;
        ++f_it;
    };
    auto fetch = [&]() {
        if (lane != 0)
            return;
        if (f_run > 0) {
            send(PL::kTileBytes);
            f_src += kStep * PL::kTileBytes;
            --f_run;
            return;
        }
        for (; f_tile < tile_end; f_tile += kStep) {
            while (f_tile >= fs.first + fs.nt)
                next_segment<T>(p, fs);
            const int tt = f_tile - fs.first;
            if (tt >= fs.v.nt)
                continue;   // an empty tile
            int pos0, end;
            tile_range<T>(fs, p.sinks, tt, pos0, end);
            const int n = min(NS, (end - pos0 + kQ4Block - 1) / kQ4Block);
            f_src = p.slot + (static_cast<long long>(fs.beta) * p.g + fs.j) * p.row_bytes +
                    static_cast<long long>(pos0 / kQ4Block) * LY::kBytes;
            send(static_cast<uint32_t>(n) * LY::kBytes);
            // the whole tiles behind it, of the same part of the segment and this run
            const int stop = min(tile_end, fs.first + (tt < fs.v.ns ? fs.v.ns : fs.v.nt)) - 1;
            f_run = f_tile < stop ? (stop - f_tile + kStep - 1) / kStep : 0;
            f_src += kStep * PL::kTileBytes;
            return;
        }
    };
    // Queries of a segment: 16 bytes (8 channels) `i` of them, a head's in neighbouring lanes.
    constexpr int kOct = D / 8;
    constexpr int kQLoads = 8 * NB * kOct;
    constexpr int kQPer = (kQLoads + PL::kThreads - 1) / PL::kThreads;   // shared runs: a thread's
    auto load_q = [&](const Segment &s, int i) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (i < kQLoads && i / kOct < p.G)
            v = *reinterpret_cast<const uint4 *>(
                p.Q + (static_cast<size_t>(s.beta) * p.h + static_cast<size_t>(s.j) * p.G) * D +
                i * 8);
        return v;
    };
    auto store_q = [&](const uint4 &v, int i) {
        const int head = i / kOct, oct = i % kOct;
        if (i >= kQLoads || head >= p.G)   // whole heads
            return;
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        // a row with a NaN or an infinity becomes NaN
        auto bad_row = [](float m) { return !(m < __int_as_float(0x7f800000)); };
        float x[8], mx = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = (i & 1) ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
            mx = fmaxf(mx, bad_row(fabsf(x[i])) ? __int_as_float(0x7f800000) : fabsf(x[i]));
        }
        // a head's kOct lanes
        const uint32_t peers = (kOct == 16 ? 0xffffu : 0xffu) << (lane & ~(kOct - 1));
#pragma unroll
        for (int m = 1; m < kOct; m <<= 1)
            mx = fmaxf(mx, __shfl_xor_sync(peers, mx, m));
        // 2^e, the largest with mx 2^e < 2^15 (within limits that keep every factor finite)
        const int e = max(-100, min(100, 14 - (static_cast<int>(__float_as_uint(mx) >> 23) - 127)));
        const float up = __int_as_float((127 + e) << 23), down = __int_as_float((127 - e) << 23);
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            y[i] = bad_row(mx) ? 0x7fff7fffu : pack_f16x2(x[2 * i] * up, x[2 * i + 1] * up);
        *reinterpret_cast<uint4 *>(const_cast<uint8_t *>(q_set) + PL::q_at(head, oct >> 2, oct & 3)) =
            make_uint4(y[0], y[1], y[2], y[3]);
        if (oct == 0)
            q_mul[head] = p.scale_log2 * kQ4Unit * down;
    };
    // A warp's own queries: all its loads, then their conversion.
    struct WarpQ {
        uint4 v[kQLoads / 32];
    };
    const int q_n = (p.G * kOct + 31) / 32;
    auto load_warp_q = [&](const Segment &s, WarpQ &q) {
#pragma unroll
        for (int i = 0; i < kQLoads / 32; ++i)
            if (i < q_n)
                q.v[i] = load_q(s, 32 * i + lane);
    };
    auto store_warp_q = [&](const WarpQ &q) {
#pragma unroll
        for (int i = 0; i < kQLoads / 32; ++i)
            if (i < q_n)
                store_q(q.v[i], 32 * i + lane);
        __syncwarp();
    };
    // The heads past the group's: zeros once.
    {
        const int n = kWarpRuns ? 32 : PL::kThreads;
        for (int i = (kWarpRuns ? lane : tid) + p.G * kOct; i < kQLoads; i += n) {
            const int head = i / kOct, oct = i % kOct;
            *reinterpret_cast<uint4 *>(const_cast<uint8_t *>(q_set) +
                                       PL::q_at(head, oct >> 2, oct & 3)) = make_uint4(0, 0, 0, 0);
            if (oct == 0)
                q_mul[head] = 1.f;
        }
    }

    grid_dependency_wait();
    grid_dependents_launch();
    if (tile_lo >= tile_hi)
        return;
    // The first queries before the first tiles: behind the whole GPU's first tiles they took 4 us.
    Segment cs = fs;
    if constexpr (kWarpRuns) {
        WarpQ q;
        load_warp_q(cs, q);
#pragma unroll
        for (int s = 0; s < R; ++s)
            fetch();
        store_warp_q(q);
    } else {
        uint4 q[kQPer];
#pragma unroll
        for (int i = 0; i < kQPer; ++i)
            q[i] = load_q(cs, tid + i * PL::kThreads);
#pragma unroll
        for (int s = 0; s < R; ++s)
            fetch();
#pragma unroll
        for (int i = 0; i < kQPer; ++i)
            store_q(q[i], tid + i * PL::kThreads);
        __syncthreads();
    }

    int it = 0;                       // this warp's tiles so far
    int tile = tile_first;
    for (int piece = tile_lo; piece < tile_hi;) {
        const int seg_end = cs.first + cs.nt;
        const int piece_end = min(seg_end, tile_hi);
        const bool last = !kWarpRuns || piece_end == tile_hi;
        Segment ns = cs;
        if (!last)
            next_segment<T>(p, ns);
        if (kWarpRuns && !last && lane * 64 < p.G * D)   // the next piece's queries to L2
            asm volatile("prefetch.global.L2 [%0];" ::"l"(
                p.Q + (static_cast<size_t>(ns.beta) * p.h + static_cast<size_t>(ns.j) * p.G) * D + lane * 64));
        // A thread's statistics are those of heads 2 tig and 2 tig + 1 (la: over its own positions);
        // O is in units of 2^-16 / up, up a power of two a head and group.
        float o[NB][2 * NG][4];
        uint32_t up[NB][NG];   // bf16, of both heads
        // A head's reference is -nm, in log2 units (products times mul are); it moves when a score exceeds
        // it.  Without one yet every score does.
        float la[NB][2], nm[NB][2], mul[NB][2];
        // The scale (bf16, twice) up to which no product of group lane % NG passes its range.
        uint32_t v_most = 0u;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int n = 0; n < 2 * NG; ++n)
                o[nb][n][0] = o[nb][n][1] = o[nb][n][2] = o[nb][n][3] = 0.f;
#pragma unroll
            for (int g = 0; g < NG; ++g)
                up[nb][g] = kQ4UpNone;
            la[nb][0] = la[nb][1] = 0.f;
            nm[nb][0] = nm[nb][1] = 3e38f;
            const float2 f = *reinterpret_cast<const float2 *>(q_mul + 8 * nb + 2 * tig);
            mul[nb][0] = f.x;
            mul[nb][1] = f.y;
        }
        const uint32_t half_sel = (gid & 1) ? 0x3244u : 0x1044u;   // a position of a pair, as fp32
        for (const int stop = kWarpRuns ? piece_end : tile_end; tile < stop; tile += kStep, ++it) {
            const int s = it % R;
            if (kWarpRuns && tile - cs.first >= cs.v.nt) {
                --it;
                continue;   // an empty tile
            }
            if (!expired && !mbar_wait(bar_full + 8 * s, (it / R) & 1)) {
                expired = true;   // the status says so; what follows is whatever the ring holds
                atomicOr(p.err, kErrWaitFull);
            }
            const uint8_t *st = smem + PL::kRing + (warp * R + s) * PL::kTileBytes;
            int pos0, end;
            tile_range<T>(cs, p.sinks, tile - cs.first, pos0, end);
            const int vis0 = (tile - cs.first < cs.v.ns ? 0 : cs.v.first) - pos0;   // visible: [vis0, vis1)
            const int vis1 = end - pos0;
            const bool edge = vis0 > 0 || vis1 < T;
            {
                // The words of V's scales are pairs of positions; two words a lane (of one group), and as a
                // position's the scales at gid (hi: gid + 8) of block b.
                auto v_word = [&](int i) {
                    const int k = lane + 32 * i;
                    return st + k / (8 * NG) * LY::kBytes + LY::kVs + k % (8 * NG) * 4;
                };
                auto v_scales = [&](int b, int hi, float (&f)[NG]) {
                    const uint8_t *at =
                        st + b * LY::kBytes + LY::kVs + ((gid >> 1) * 2 + hi) * NG * 4;
                    uint32_t w[NG];
                    if constexpr (NG == 4) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(at);
                        w[0] = x.x;
                        w[1] = x.y;
                        w[2] = x.z;
                        w[3] = x.w;
                    } else {
                        const uint2 x = *reinterpret_cast<const uint2 *>(at);
                        w[0] = x.x;
                        w[1] = x.y;
                    }
#pragma unroll
                    for (int g = 0; g < NG; ++g)
                        f[g] = __uint_as_float(__byte_perm(w[g], 0u, half_sel));
                };
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
                            *reinterpret_cast<const uint4 *>(q_set + PL::q_at(8 * nb + gid, g, tig));
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
                            float t[4];
                            mma_f16_zero(t, a[0], a[1], a[2], a[3], q[nb].x, q[nb].y);
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
                    // Positions outside [vis0, vis1) hold anything, NaN scales among it: V's become zeros, in
                    // place (the stage's next copy comes after the fence).
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int k = lane + 32 * i, at = k % (8 * NG);
                        const int r = 16 * (k / (8 * NG)) + 8 * (at / NG & 1) + 2 * (at / (2 * NG));
                        uint16_t *pair =
                            reinterpret_cast<uint16_t *>(const_cast<uint8_t *>(v_word(i)));
                        if (r < vis0 || r >= vis1)
                            pair[0] = 0;
                        if (r + 1 < vis0 || r + 1 >= vis1)
                            pair[1] = 0;
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                // ---- online softmax (base 2), references and powers of two moved rarely ----
                float mx[NB][2];
                bool raise = false;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    mx[nb][0] = mx[nb][1] = NEG_INF;
#pragma unroll
                    for (int b = 0; b < NS; ++b) {
                        mx[nb][0] = fmaxf(mx[nb][0], fmaxf(sc[b][nb][0], sc[b][nb][2]));
                        mx[nb][1] = fmaxf(mx[nb][1], fmaxf(sc[b][nb][1], sc[b][nb][3]));
                    }
                    raise |= fmaf(mx[nb][0], mul[nb][0], nm[nb][0]) > 0.f ||
                             fmaf(mx[nb][1], mul[nb][1], nm[nb][1]) > 0.f;
                }
                // whether a product of weight and scale may pass its range (bf16 numbers >= 0 are ordered like
                // their bits, NaN last)
                const bool may_pass =
                    __vimax3_u16x2(*reinterpret_cast<const uint32_t *>(v_word(0)),
                                   *reinterpret_cast<const uint32_t *>(v_word(1)), v_most) != v_most;
                if (__any_sync(0xffffffffu, raise || may_pass)) {
                    float alpha[NB][2], lift[NB][2];   // of the sums so far; of the powers of two
                    uint32_t x[NB][NG];   // the largest products, two heads' leading 16 bits
                    bool move = raise;
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            float y = mx[nb][i];
                            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 4));
                            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 8));
                            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 16));
                            alpha[nb][i] = lift[nb][i] = 1.f;
                            if (fmaf(y, mul[nb][i], nm[nb][i]) > 0.f) {
                                const float nm_new = fmaf(-y, mul[nb][i], -kQ4LazyMax);
                                const float by = nm_new - nm[nb][i];
                                alpha[nb][i] = fast_exp2(by);   // 0 where there was none
                                // what has been summed keeps its size: floor(-by), 2^120 at most
                                lift[nb][i] =
                                    __int_as_float((127 + static_cast<int>(fminf(-by, 120.f))) << 23);
                                nm[nb][i] = nm_new;
                            }
                            la[nb][i] *= alpha[nb][i];
                        }
                        float y[NG][2];   // the largest products (NaN ones move nothing)
#pragma unroll
                        for (int g = 0; g < NG; ++g)
                            y[g][0] = y[g][1] = 0.f;
#pragma unroll
                        for (int b = 0; b < NS; ++b)
#pragma unroll
                            for (int hi = 0; hi < 2; ++hi) {
                                float f[NG];
                                v_scales(b, hi, f);
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    const float w = fast_exp2(
                                        fmaf(sc[b][nb][2 * hi + i], mul[nb][i], nm[nb][i]));
#pragma unroll
                                    for (int g = 0; g < NG; ++g)
                                        y[g][i] = fmaxf(y[g][i], w * f[g]);
                                }
                            }
#pragma unroll
                        for (int g = 0; g < NG; ++g) {
                            x[nb][g] = __byte_perm(__float_as_uint(y[g][0]), __float_as_uint(y[g][1]), 0x7632);
                            move |= y[g][0] * bf16_lo(up[nb][g]) >= kQ4ProductMost ||
                                    y[g][1] * bf16_hi(up[nb][g]) >= kQ4ProductMost;
                        }
                    }
                    if (__any_sync(0xffffffffu, move)) {
#pragma unroll
                        for (int g = 0; g < NG; ++g) {
                            float m = 0.f;   // the largest power of two of the lane's heads
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb) {
                                uint32_t z = x[nb][g];
                                z = __vmaxu2(z, __shfl_xor_sync(0xffffffffu, z, 4));
                                z = __vmaxu2(z, __shfl_xor_sync(0xffffffffu, z, 8));
                                z = __vmaxu2(z, __shfl_xor_sync(0xffffffffu, z, 16));
                                float to[2];
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    const float y = i == 0 ? bf16_lo(z) : bf16_hi(z);
                                    const float u = i == 0 ? bf16_lo(up[nb][g]) : bf16_hi(up[nb][g]);
                                    to[i] = fminf(u * lift[nb][i], 0x1p126f);
                                    if (y * to[i] >= kQ4ProductMost)   // 2^(kQ4ProductTop - floor(log2 y))
                                        to[i] = __uint_as_float(
                                            (254u + kQ4ProductTop - (__float_as_uint(y) >> 23)) << 23);
                                    const float f = alpha[nb][i] * (to[i] * reciprocal2(u));
#pragma unroll
                                    for (int n = 0; n < 2; ++n) {
                                        o[nb][2 * g + n][i] *= f;
                                        o[nb][2 * g + n][2 + i] *= f;
                                    }
                                    m = fmaxf(m, to[i]);
                                }
                                up[nb][g] = __byte_perm(__float_as_uint(to[0]), __float_as_uint(to[1]), 0x7632);
                            }
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
                            if (lane % NG == g)   // a power of two
                                v_most = (__float_as_uint(kQ4ProductMost * reciprocal2(m)) >> 16) * 0x10001u;
                        }
                    }
                }
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    const float2 mul2 = make_float2(mul[nb][0], mul[nb][1]);
                    const float2 nm2 = make_float2(nm[nb][0], nm[nb][1]);
                    float2 l2 = make_float2(la[nb][0], la[nb][1]);
#pragma unroll
                    for (int b = 0; b < NS; ++b)
#pragma unroll
                        for (int hi = 0; hi < 2; ++hi) {
                            float *x = sc[b][nb] + 2 * hi;
                            const float2 y = __ffma2_rn(make_float2(x[0], x[1]), mul2, nm2);
                            x[0] = fast_exp2(y.x);
                            x[1] = fast_exp2(y.y);
                            l2 = __fadd2_rn(l2, make_float2(x[0], x[1]));
                        }
                    la[nb][0] = l2.x;
                    la[nb][1] = l2.y;
                }
                // ---- O += V^T (s P)^T ----
#pragma unroll
                for (int b = 0; b < NS; ++b) {
                    const uint8_t *blk = st + b * LY::kBytes;
                    // weights times scales, in fp32, rounded once, [hi][group]
                    uint32_t pb[NB][2 * NG];
                    float f[2][NG];
                    v_scales(b, 0, f[0]);
                    v_scales(b, 1, f[1]);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int k = 0; k < 2 * NG; ++k) {
                            const int hi = k / NG, g = k % NG;
                            const float2 w = make_float2(sc[b][nb][2 * hi], sc[b][nb][2 * hi + 1]);
                            const float2 u = make_float2(bf16_lo(up[nb][g]), bf16_hi(up[nb][g]));
                            const float2 x = __fmul2_rn(__fmul2_rn(w, make_float2(f[hi][g], f[hi][g])), u);
                            pb[nb][k] = movmatrix_trans(pack_f16x2(x.x, x.y));
                        }
                    uint32_t vw[2 * NG];   // [th][group]
#pragma unroll
                    for (int q = 0; q < 2 * NG / 4; ++q) {
                        const uint4 w =
                            *reinterpret_cast<const uint4 *>(blk + LY::kV + q * 512 + lane * 16);
                        vw[4 * q] = w.x;
                        vw[4 * q + 1] = w.y;
                        vw[4 * q + 2] = w.z;
                        vw[4 * q + 3] = w.w;
                    }
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        const uint32_t w0 = vw[g], w1 = vw[NG + g];
                        const uint32_t a[8] = {q4_pair(w0, 0), q4_pair(w0, 1), q4_pair(w1, 0),
                                               q4_pair(w1, 1), q4_pair(w0, 2), q4_pair(w0, 3),
                                               q4_pair(w1, 2), q4_pair(w1, 3)};
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) {
                            mma_f16(o[nb][2 * g], a[0], a[1], a[2], a[3], pb[nb][g], pb[nb][NG + g]);
                            mma_f16(o[nb][2 * g + 1], a[4], a[5], a[6], a[7], pb[nb][g], pb[nb][NG + g]);
                        }
                    }
                }
            }
            __syncwarp();
            fetch();   // into the stage just read
        }

        // ---- end of the piece ----
        const int G = p.G, seg = cs.beta * p.g + cs.j;
        const bool whole = piece == cs.first && piece_end == seg_end;
        const size_t rec = static_cast<size_t>(seg) + run;
        __nv_bfloat16 *ob =
            p.out + (static_cast<size_t>(cs.beta) * p.h + static_cast<size_t>(cs.j) * G) * D;
        // the runs that hold the segment
        const int c0 = cta_of_tile(cs.first, N, P), c1 = cta_of_tile(seg_end - 1, N, P);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                la[nb][i] += __shfl_xor_sync(0xffffffffu, la[nb][i], 4);
                la[nb][i] += __shfl_xor_sync(0xffffffffu, la[nb][i], 8);
                la[nb][i] += __shfl_xor_sync(0xffffffffu, la[nb][i], 16);
            }
        // Four channels of head 2 tig + i and group g: the piece's sums, over its weights' (inv: 1 / la) before
        // they leave the units of codes and scales, lest they pass fp32's range.
        auto mean4 = [&](int nb, int g, int i, float inv) {
            const float u = i == 0 ? bf16_lo(up[nb][g]) : bf16_hi(up[nb][g]);
            const float down = reciprocal2(u);
            inv *= kQ4Unit;
            return make_float4(o[nb][2 * g][i] * inv * down, o[nb][2 * g][2 + i] * inv * down,
                               o[nb][2 * g + 1][i] * inv * down, o[nb][2 * g + 1][2 + i] * inv * down);
        };
        // Merges the segment's records, in their order, by the threads t of n: C times four columns of K
        // records a thread in flight (one round trip to L2 after another otherwise: 6 us at the end of
        // a launch).
        auto merge = [&](int t, int n, auto c_, auto k_) {
            constexpr int C = decltype(c_)::value, K = decltype(k_)::value;
            const int np = c1 - c0 + 1;
            const size_t rec0 = static_cast<size_t>(seg) + c0;
            for (int i0 = 4 * t; i0 < G * D; i0 += 4 * n * C) {
                float mx[C], tot[C];
                float4 a[C];
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    mx[c] = NEG_INF;
                    tot[c] = 0.f;
                    a[c] = make_float4(0.f, 0.f, 0.f, 0.f);
                }
                for (int k0 = 0; k0 < np; k0 += K) {
                    float l[K][C];
                    float4 x[K][C];
#pragma unroll
                    for (int k = 0; k < K; ++k)
#pragma unroll
                        for (int c = 0; c < C; ++c) {
                            const int i = i0 + 4 * n * c;
                            l[k][c] = NEG_INF;
                            x[k][c] = make_float4(0.f, 0.f, 0.f, 0.f);
                            if (k0 + k < np && i < G * D) {
                                l[k][c] = __ldcg(&p.part_lse[(rec0 + k0 + k) * G + i / D]);
                                x[k][c] = __ldcg(reinterpret_cast<const float4 *>(
                                    p.part_o + (rec0 + k0 + k) * G * D + i));
                            }
                        }
#pragma unroll
                    for (int c = 0; c < C; ++c) {
                        float m_new = mx[c];
#pragma unroll
                        for (int k = 0; k < K; ++k)
                            m_new = fmaxf(m_new, l[k][c]);
                        // (a run may hold empty tiles of the segment alone: no weight at all yet)
                        const float base = m_new == NEG_INF ? 0.f : m_new;
                        const float down = fast_exp2(mx[c] - base);   // 0 before the first weight
                        mx[c] = m_new;
                        tot[c] *= down;
                        a[c].x *= down;
                        a[c].y *= down;
                        a[c].z *= down;
                        a[c].w *= down;
#pragma unroll
                        for (int k = 0; k < K; ++k) {
                            const float f = fast_exp2(l[k][c] - base);   // 0 past the records
                            tot[c] += f;
                            a[c].x = fmaf(f, x[k][c].x, a[c].x);
                            a[c].y = fmaf(f, x[k][c].y, a[c].y);
                            a[c].z = fmaf(f, x[k][c].z, a[c].z);
                            a[c].w = fmaf(f, x[k][c].w, a[c].w);
                        }
                    }
                }
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int i = i0 + 4 * n * c;
                    const float inv = fast_rcp(tot[c]);
                    if (i < G * D)
                        *reinterpret_cast<uint2 *>(ob + i) =
                            make_uint2(pack_bf16x2(a[c].x * inv, a[c].y * inv),
                                       pack_bf16x2(a[c].z * inv, a[c].w * inv));
                }
            }
        };
        if constexpr (kWarpRuns) {
            // The warp holds the piece's sums: four channels of a head and group a lane.
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int head = 8 * nb + 2 * tig + i;
                    if (head < G) {
                        // (a piece of empty tiles: zeros, with the weight 2^-inf)
                        const float inv = la[nb][i] == 0.f ? 0.f : fast_rcp(la[nb][i]);
                        const size_t at = static_cast<size_t>(head) * D + gid * 4;
#pragma unroll
                        for (int g = 0; g < NG; ++g) {
                            const float4 v = mean4(nb, g, i, inv);
                            if (whole)
                                *reinterpret_cast<uint2 *>(ob + at + 32 * g) =
                                    make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
                            else
                                *reinterpret_cast<float4 *>(p.part_o + rec * G * D + at + 32 * g) = v;
                        }
                        if (!whole && gid == 0)
                            p.part_lse[rec * G + head] = fast_log2(la[nb][i]) - nm[nb][i];
                    }
                }
            if (!whole && !p.deferred_merge) {
                // The warp that finishes a segment last merges its records.
                __syncwarp();
                unsigned prev = 0;
                if (lane == 0)
                    prev = atomic_add_acq_rel_gpu(&p.counters[seg], 1u);
                prev = __shfl_sync(0xffffffffu, prev, 0);
                __syncwarp();
                if (prev == static_cast<unsigned>(c1 - c0)) {
                    merge(lane, 32, std::integral_constant<int, 4>{},
                          std::integral_constant<int, 4>{});
                    if (lane == 0)
                        p.counters[seg] = 0u;
                }
            }
            piece = piece_end;
            cs = ns;
            if (!last) {
                WarpQ q;
                load_warp_q(cs, q);
                store_warp_q(q);
            }
            continue;
        }
        // Shared runs: the warps' sums are merged, 8 heads at a time.
        float *raw = reinterpret_cast<float *>(smem + PL::kRaw);          // [kWarps][8][kRow]
        float *st_m = reinterpret_cast<float *>(smem + PL::kStat);        // [8 NB][kWarps]
        float *st_l = st_m + 8 * NB * NW;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            if (nb > 0 && G <= 8 * nb)
                break;
            if (nb > 0)
                __syncthreads();   // the sums of the heads before have been read
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float *dst = raw + (warp * 8 + 2 * tig + i) * PL::kRow + gid * 4;
                // (a warp without a tile: zeros, with the weight 0)
                const float inv = la[nb][i] == 0.f ? 0.f : fast_rcp(la[nb][i]);
#pragma unroll
                for (int g = 0; g < NG; ++g)
                    *reinterpret_cast<float4 *>(dst + g * 32) = mean4(nb, g, i, inv);
                if (gid == 0) {
                    st_m[(8 * nb + 2 * tig + i) * NW + warp] = -nm[nb][i];
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
                float ls = 0.f, weight[NW];
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    weight[w] = st_l[(8 * nb + row) * NW + w] *
                                fast_exp2(st_m[(8 * nb + row) * NW + w] - ms);
                    ls += weight[w];
                }
                const float inv = fast_rcp(ls);
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    const float f = weight[w] * inv;
                    const float4 x =
                        *reinterpret_cast<const float4 *>(raw + (w * 8 + row) * PL::kRow + e);
                    v.x = fmaf(f, x.x, v.x);
                    v.y = fmaf(f, x.y, v.y);
                    v.z = fmaf(f, x.z, v.z);
                    v.w = fmaf(f, x.w, v.w);
                }
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
        if (!whole && !p.deferred_merge) {
            // The CTA that finishes a segment last merges its records.
            __syncthreads();
            if (tid == 0)
                flags[0] = atomic_add_acq_rel_gpu(&p.counters[seg], 1u) ==
                           static_cast<unsigned>(c1 - c0);
            __syncthreads();
            if (flags[0]) {
                merge(tid, PL::kThreads, std::integral_constant<int, 1>{},
                      std::integral_constant<int, 8>{});
                if (tid == 0)
                    p.counters[seg] = 0u;
            }
        }
        break;
    }
    // No copy may still be in flight when the CTA exits (after an expired wait).
    if (lane == 0 && expired) {
        for (int k = f_it > R ? f_it - R : 0; k < f_it; ++k)
            if (!mbar_wait(bar_full + 8 * (k % R), (k / R) & 1))
                atomicOr(p.err, kErrDrain);
    }
}

struct Variant {
    const void *fn;
    size_t smem;
};

template <int D, int NB, bool kWarpRuns>
Variant variant()
{
    return {reinterpret_cast<const void *>(&q4_decode_kernel<D, NB, kWarpRuns>),
            static_cast<size_t>(Q4Plan<D, NB, kWarpRuns>::kBytes)};
}

template <int D, int NB>
Variant variant(bool warp_runs)
{
    return warp_runs ? variant<D, NB, true>() : variant<D, NB, false>();
}

Variant find_variant(int d, int group, bool warp_runs)
{
    if (d == 64)
        return group <= 8 ? variant<64, 1>(warp_runs) : variant<64, 2>(warp_runs);
    return group <= 8 ? variant<128, 1>(warp_runs) : variant<128, 2>(warp_runs);
}

}  // namespace

cudaError_t prepare_q4_decode(int d, int group, int *ctas_per_sm)
{
    *ctas_per_sm = 1 << 30;
    for (const bool warp_runs : {false, true}) {
        const Variant v = find_variant(d, group, warp_runs);
        cudaError_t e = cudaFuncSetAttribute(v.fn, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             static_cast<int>(v.smem));
        int n = 0;
        if (e == cudaSuccess)
            e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, v.fn, q4_warps(d, group) * 32,
                                                              v.smem);
        if (e != cudaSuccess)
            return e;
        *ctas_per_sm = n < *ctas_per_sm ? n : *ctas_per_sm;
    }
    return cudaSuccess;
}

cudaError_t launch_q4_decode(int d, int grid, bool warp_runs, const Q4DecodeParams &p,
                             cudaStream_t stream)
{
    const Variant v = find_variant(d, p.G, warp_runs);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(grid));
    cfg.blockDim = dim3(static_cast<unsigned>(q4_warps(d, p.G) * 32));
    cfg.dynamicSmemBytes = v.smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    void *args[] = {const_cast<Q4DecodeParams *>(&p)};
    return cudaLaunchKernelExC(&cfg, v.fn, args);
}

}  // namespace mlkv
