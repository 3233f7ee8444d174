// Decode attention over pieces of a cache for GB300: the common core of three calls.
//
//   suffix    a sequence's own positions, merged with the records of a prefix that other sequences share
//   joined    a prefix's positions and then the sequence's own, end to end
//   groups    suffixes, and beside them the prefix's positions for as many sequences as have 16 heads together
//   blocks    the blocks of 64 positions listed for every (sequence, KV head)
//   weights   all positions, every score stored on the way (weights_kernel turns them into weights)
//
// For the G query heads of one KV head, s_u = q k_u log2(e) / sqrt(d), m = max s, o = sum 2^(s_u - m) v_u / l,
// l = sum 2^(s_u - m), in one pass with a running m (Eqs. 2-3 of arXiv 2406.09297 with the maps of Eqs. 15
// and 18).  A piece's result is the record (o, m + log2 l); records merge as
//   o = sum_c 2^(lse_c - M) o_c / sum_c 2^(lse_c - M),   M = max_c lse_c.
//
// A CTA is one piece: a producer warp brings tiles of 64 keys and values through a ring by TMA.  The consumer warps
// take the tiles in turn, one a tile of 64 channels, two of 32 keys each a tile of 128, with sums of their own that meet
// in shared memory at the end.  S^T = K Q^T and O^T += V^T P by mma.sync m16n8k16, heads as columns: eight heads
// take half the products of heads as rows.  A segment's records are merged, in their order, by the CTA that
// finishes it last or, where there are many, by a launch of their own: outputs do not depend on which CTA is last.
// Bound by the bytes of keys and values (4 d flops for each 4 d bytes and head leave the tensor cores idle): two CTAs
// an SM keep 192 KB in flight, three times what the latency of HBM needs.  32 sequences of 8192 positions, 8 KV heads
// of 128 with their scores, 160.6 us, 6.7 TB/s; 32 times 64 blocks of 64, the same heads, 77 us, 7.0 TB/s.
#include "mlkv_device.cuh"
#include "mlkv_long.h"

namespace mlkv {
namespace {

constexpr int T = kBlock;

template <int D>
struct PiecePlan {
    static constexpr int kTile = T * D * 2;            // K or V of a tile
    static constexpr int kStages = D == 64 ? 6 : 3;
    // Consumer warps: the same ones for a stage throughout.  (A stage's barrier tells two of its phases apart, so
    // whoever waits for one has to have seen the one before.)
    static constexpr int kPerStage = D == 64 ? 1 : 2;
    static constexpr int kWarps = kStages * kPerStage;
    static constexpr int kKeys = T / kPerStage;        // of a warp and tile
    static constexpr int kThreads = (kWarps + 1) * 32;
    static constexpr int kBars = kStages * 2 * kTile;  // full[], empty[]
    static constexpr int kML = kBars + 2 * 8 * kStages;   // float [kWarps][2][16]
    static constexpr int kFlag = kML + kWarps * 2 * 16 * 4;
    static constexpr int kBytes = kFlag + 16;
    static constexpr int kRow = D + 4;                 // floats of a row of a warp's sums
    static_assert(kWarps * 16 * kRow * 4 <= kBars, "sums fit in the ring");
    static_assert(2 * (kBytes + 1024) <= 228 * 1024, "two CTAs an SM");
};

// Room for merge weights, in the ring.
template <int D>
constexpr int max_records(int G)
{
    return PiecePlan<D>::kBars / (4 * G);
}

__device__ __forceinline__ float neg_inf() { return -__int_as_float(0x7f800000); }

struct Piece {
    int beta, j, seg, index, count, t0, t1, L;   // beta: the query row
    int rows;      // heads of the piece's tile
    int out_row;   // of out
    int unit, place, prefix, chunk;              // kPieceGroups: a unit (else 0), its place, prefix and chunk
};

// Row of Q and out, and sequence, of a query row.
// (only what runs over prefixes has scattered rows, kPieceGroups none)
template <int kMode>
__device__ __forceinline__ int q_row_of(const PieceArgs<kMode> &p, int i)
{
    if constexpr (kMode == kPieceSuffix || kMode == kPieceJoined)
        return p.scattered ? p.q_row[i] : i;
    return i;
}
template <int kMode>
__device__ __forceinline__ int row_seq(const PieceArgs<kMode> &p, int i)
{
    if constexpr (kMode == kPieceSuffix || kMode == kPieceJoined)
        return p.scattered ? p.seq[i] : i;
    return i;
}

// The i-th row as the pieces are laid out.
__device__ __forceinline__ int row_at(const PieceBase &p, int i) { return p.ordered ? p.order[i] : i; }

// The records of the prefix that the row merges, and their first one for KV head j.
template <int kMode>
__device__ __forceinline__ int prefix_records(const PieceArgs<kMode> &p, int i)
{
    if constexpr (kMode == kPieceSuffix || kMode == kPieceGroups)
        return p.pre_n[i];
    return 0;
}
template <int kMode>
__device__ __forceinline__ size_t prefix_record(const PieceArgs<kMode> &p, int i, int j)
{
    if constexpr (kMode == kPieceSuffix || kMode == kPieceGroups)
        return p.pre_n[i] > 0 ? (static_cast<size_t>(p.pre_place[i]) * p.g + j) * p.pre_chunks : 0;
    return 0;
}

template <int kMode>
__device__ __forceinline__ Piece piece_of(const PieceArgs<kMode> &p)
{
    Piece x;
    x.unit = x.place = x.prefix = x.chunk = 0;
    x.rows = p.G;
    int c = static_cast<int>(blockIdx.x);
    if constexpr (kMode == kPieceGroups) {
        if (c < p.n_units) {
            const uint32_t u = p.units[c];
            x.unit = 1;
            x.prefix = static_cast<int>(u & 0x3ffu);
            x.chunk = static_cast<int>((u >> 10) & 0xffu);
            x.j = static_cast<int>((u >> 18) & 0xffu);
            x.rows = (static_cast<int>(u >> 26) + 1) * p.G;
            x.place = p.unit_place[c];
            x.beta = x.seg = x.index = x.out_row = 0;
            x.count = 1;
            x.L = p.prefix_len[x.prefix];
            x.t0 = x.chunk * p.unit_tiles;
            x.t1 = min((x.L + T - 1) / T, x.t0 + p.unit_tiles);
            return x;
        }
        c -= p.n_units;
    }
    int lo = 0, hi = p.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.first[mid] <= c)
            lo = mid;
        else
            hi = mid - 1;
    }
    x.beta = row_at(p, lo);
    x.L = p.seq_len[x.beta];
    const int nt = piece_tiles<kMode>(p, x.beta);
    x.count = (nt + p.tiles - 1) / p.tiles;
    const int rel = c - p.first[lo];
    x.j = rel / x.count;
    x.index = rel - x.j * x.count;
    x.seg = x.beta * p.g + x.j;
    x.out_row = q_row_of<kMode>(p, x.beta);
    x.t0 = x.index * p.tiles;
    x.t1 = min(nt, x.t0 + p.tiles);
    return x;
}

// Merges the segment's records (its own pieces', from own0 on, then the prefix's n_pre from pre0 on) into out: the
// weights first, then the sums in the records' order.  s_w: room for a row of G floats a record, and one more.
template <int D>
__device__ void merge_records(const PieceBase &p, const Piece &x, size_t own0, int n_pre, size_t pre0, float *s_w,
                              int tid, int n_threads)
{
    const int G = p.G, n_own = x.count, n = n_own + n_pre;
    for (int i = tid; i < n * G; i += n_threads)
        s_w[i] = i < n_own * G ? __ldcg(p.part_lse + own0 * G + i)
                               : __ldcg(p.pre_lse + pre0 * G + (i - n_own * G));
    asm volatile("bar.sync 1, %0;" ::"r"(n_threads) : "memory");
    if (tid < G) {
        float mx = neg_inf();
        for (int k = 0; k < n; ++k)
            mx = fmaxf(mx, s_w[k * G + tid]);
        float tot = 0.f;
        for (int k = 0; k < n; ++k) {
            // (a NaN of a record goes on into the sum; without anything visible every weight is 0)
            const float lse = s_w[k * G + tid];
            const float w = lse == neg_inf() ? 0.f : fast_exp2(lse - mx);
            s_w[k * G + tid] = w;
            tot += w;
        }
        s_w[n * G + tid] = tot == 0.f ? 0.f : 1.f / tot;
    }
    asm volatile("bar.sync 1, %0;" ::"r"(n_threads) : "memory");
    __nv_bfloat16 *ob = p.out + (static_cast<size_t>(x.out_row) * p.h + static_cast<size_t>(x.j) * G) * D;
    for (int i = tid * 4; i < G * D; i += n_threads * 4) {
        const int row = i / D;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int U = 8;
        for (int k0 = 0; k0 < n; k0 += U) {
            float4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int k = k0 + u;
                const float *rec = k < n_own ? p.part_o + (own0 + k) * G * D
                                             : p.pre_o + (pre0 + (k - n_own)) * G * D;
                v[u] = k < n ? __ldcg(reinterpret_cast<const float4 *>(rec + i))
                             : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int k = k0 + u;
                const float w = k < n ? s_w[k * G + row] : 0.f;
                if (w != 0.f) {
                    acc.x = fmaf(w, v[u].x, acc.x);
                    acc.y = fmaf(w, v[u].y, acc.y);
                    acc.z = fmaf(w, v[u].z, acc.z);
                    acc.w = fmaf(w, v[u].w, acc.w);
                }
            }
        }
        const float inv = s_w[n * G + row];
        uint2 w2;
        w2.x = pack_bf16x2(acc.x * inv, acc.y * inv);
        w2.y = pack_bf16x2(acc.z * inv, acc.w * inv);
        *reinterpret_cast<uint2 *>(ob + i) = w2;
    }
}

// NH: groups of eight query heads, 1 or 2.
template <int D, int kMode, int NH>
__global__ void __launch_bounds__(PiecePlan<D>::kThreads, 2)
    piece_kernel(const __grid_constant__ CUtensorMap tmap, const __grid_constant__ CUtensorMap tmap_prefix,
                 const __grid_constant__ PieceArgs<kMode> p)
{
    using PL = PiecePlan<D>;
    constexpr int S = PL::kStages, kWarps = PL::kWarps;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sbase = smem_addr(smem);
    const uint32_t bar_full = sbase + PL::kBars, bar_empty = bar_full + 8 * S;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *flag = reinterpret_cast<volatile int *>(smem + PL::kFlag);
    // The producer sets the barriers up and goes on to its first tiles; the consumers wait for that, behind the
    // loads of their queries.
    if (threadIdx.x == kWarps * 32) {
        prefetch_tensormap(&tmap);
        for (int s = 0; s < S; ++s) {
            mbar_init(bar_full + 8 * s, 1);
            mbar_init(bar_empty + 8 * s, PL::kPerStage);
        }
        flag[0] = 0;   // a wait gave up
        fence_barrier_init();
    }
    const bool early = kMode == kPieceSuffix && p.early;
    const bool group = kMode == kPieceGroups;
    if (!early)
        grid_dependency_wait();
    grid_dependents_launch();
    const Piece x = piece_of<kMode>(p);
    const int *list = kMode == kPieceBlocks ? p.blocks + static_cast<size_t>(x.seg) * p.n_blocks : nullptr;
    // (kPieceJoined: the prefix's tiles come first, then the sequence's own)
    int pre_len = 0;
    if constexpr (kMode == kPieceJoined)
        pre_len = p.pre_len[x.beta];
    const int n_joined = (pre_len + T - 1) / T;
    // Block of tile t, or -1: none (kPieceBlocks); 32 of a list at a time, a lane each.
    int listed = -1, listed_at = -1;
    auto block_of = [&](int t) {
        if (kMode != kPieceBlocks)
            return kMode == kPieceJoined && t >= n_joined ? t - n_joined : t;
        const int at = t & ~31;
        if (at != listed_at) {
            listed = at + lane < x.t1 ? list[at + lane] : -1;
            listed_at = at;
        }
        const int blk = __shfl_sync(0xffffffffu, listed, t & 31);
        return blk >= 0 && blk < (x.L + T - 1) / T ? blk : -1;
    };

    if (warp == kWarps) {
        __syncwarp();
        asm volatile("bar.arrive 2, %0;" ::"n"(PL::kThreads) : "memory");
        // ------------------------------------ producer ------------------------------------------
        const int zk = ((p.slot * 2 + 0) * p.b + row_seq<kMode>(p, x.beta)) * p.g + x.j, zv = zk + p.b * p.g;
        int zk_pre = 0, zv_pre = 0;
        if constexpr (kMode == kPieceJoined || kMode == kPieceGroups) {
            zk_pre = (p.slot * 2 * p.prefix_b +
                      (group ? x.prefix : static_cast<int>(p.pre_place[x.beta]))) * p.g + x.j;
            zv_pre = zk_pre + p.prefix_b * p.g;
        }
        int idx = 0;
        for (int t = x.t0; t < x.t1; ++t) {
            const int blk = block_of(t);
            if (blk < 0)
                continue;
            const int s = idx % S;
            int ok = 1;
            if (lane == 0) {
                if (idx >= S && !mbar_wait(bar_empty + 8 * s, ((idx / S) & 1) ^ 1)) {
                    flag[0] = 1;
                    atomicOr(p.err, kErrWaitEmpty);
                }
                ok = !flag[0];
                if (ok) {
                    const uint32_t fb = bar_full + 8 * s, dst = sbase + s * 2 * PL::kTile;
                    mbar_arrive_expect_tx(fb, 2 * PL::kTile);
                    const bool pre = (kMode == kPieceJoined && t < n_joined) || (group && x.unit);
                    const CUtensorMap *map = pre ? &tmap_prefix : &tmap;
#pragma unroll
                    for (int sub = 0; sub < D / 64; ++sub)
                        tma_load_3d(dst + sub * T * 128, map, fb, sub * 64, blk * T, pre ? zk_pre : zk);
#pragma unroll
                    for (int sub = 0; sub < D / 64; ++sub)
                        tma_load_3d(dst + PL::kTile + sub * T * 128, map, fb, sub * 64, blk * T,
                                    pre ? zv_pre : zv);
                }
            }
            if (!__shfl_sync(0xffffffffu, ok, 0))
                break;
            ++idx;
        }
        // No copy may still be in flight when the CTA exits.
        if (lane == 0)
            for (int k = idx > S ? idx - S : 0; k < idx; ++k)
                if (!mbar_wait(bar_full + 8 * (k % S), (k / S) & 1))
                    atomicOr(p.err, kErrDrain);
        return;
    }

    // -------------------------------------- consumers -------------------------------------------
    // Transposed: S^T = K Q^T has the warp's keys as rows and the heads as columns, O^T = V^T P the channels as rows, so
    // that up to eight heads take half the products of heads as 16 rows.  A lane holds heads 2 q and 2 q + 1 of a group
    // of eight (q = lane % 4), keys or channels lane / 4 and 8 more of 16.
    constexpr int M = PL::kKeys / 16;
    const int half = warp % PL::kPerStage * PL::kKeys;   // the warp's first key of a tile
    uint32_t qf[D / 16][NH][2];   // columns n = lane / 4
    {
#pragma unroll
        for (int nh = 0; nh < NH; ++nh) {
            const int head = nh * 8 + (lane >> 2);   // of the tile's rows
            int row = q_row_of<kMode>(p, x.beta), at = head;
            if constexpr (kMode == kPieceGroups)
                if (x.unit && head < x.rows) {
                    row = p.place_row[x.place + head / p.G];
                    at = head % p.G;
                }
            const __nv_bfloat16 *q =
                p.Q + (static_cast<size_t>(row) * p.h + static_cast<size_t>(x.j) * p.G + at) * D + (lane & 3) * 2;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    qf[kk][nh][i] =
                        head < x.rows ? *reinterpret_cast<const uint32_t *>(q + kk * 16 + i * 8) : 0u;
        }
    }
    asm volatile("bar.sync 2, %0;" ::"n"(PL::kThreads) : "memory");
    float m[NH][2], l[NH][2];
    float o[D / 16][NH][4];
#pragma unroll
    for (int nh = 0; nh < NH; ++nh) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            m[nh][i] = neg_inf();
            l[nh][i] = 0.f;
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                o[c][nh][e] = 0.f;
    }
    const int mi = lane >> 3, mr = lane & 7;   // ldmatrix: matrix and row of this lane's address
    int idx = 0;
    bool ok = true;
    for (int t = x.t0; t < x.t1; ++t) {
        const int blk = block_of(t);
        if (blk < 0)
            continue;
        const int mine = idx++;
        const int s = mine % S;
        if (s != warp / PL::kPerStage)
            continue;
        if (!mbar_wait(bar_full + 8 * s, (mine / S) & 1))
            ok = false;
        if (__any_sync(0xffffffffu, !ok || flag[0])) {
            if (lane == 0) {
                flag[0] = 1;
                atomicOr(p.err, kErrWaitFull);
            }
            ok = false;
            break;
        }
        const uint32_t kb = sbase + s * 2 * PL::kTile, vb = kb + PL::kTile;
        float sc[M][NH][4];
#pragma unroll
        for (int n = 0; n < M; ++n)
#pragma unroll
            for (int nh = 0; nh < NH; ++nh)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sc[n][nh][e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
            for (int n = 0; n < M; ++n) {
                uint32_t a[4];
                ldsm_x4(kb + swz<T>(half + n * 16 + (mi & 1) * 8 + mr, kk * 2 + (mi >> 1)), a[0], a[1], a[2], a[3]);
#pragma unroll
                for (int nh = 0; nh < NH; ++nh)
                    mma_bf16_16816(sc[n][nh], a, qf[kk][nh][0], qf[kk][nh][1]);
            }
        // visible of the warp's keys; kKeys or more: all
        const int lim = (kMode == kPieceJoined && t < n_joined ? pre_len : x.L) - blk * T - half;
#pragma unroll
        for (int n = 0; n < M; ++n)
#pragma unroll
            for (int nh = 0; nh < NH; ++nh)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sc[n][nh][e] *= p.scale_log2;
        if (lim < PL::kKeys) {
#pragma unroll
            for (int n = 0; n < M; ++n)
#pragma unroll
                for (int nh = 0; nh < NH; ++nh)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (n * 16 + (lane >> 2) + (e >> 1) * 8 >= lim)
                            sc[n][nh][e] = neg_inf();
            // Values behind the sequence's end may be anything: their weight 0 takes zeros.
            const int from = max(lim, 0);
            for (int i = lane; i < (PL::kKeys - from) * (D / 8); i += 32)
                *reinterpret_cast<uint4 *>(smem + (vb - sbase) +
                                           swz<T>(half + from + i / (D / 8), i % (D / 8))) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
            __syncwarp();
        }
        if (kMode == kPieceWeights) {
#pragma unroll
            for (int nh = 0; nh < NH; ++nh)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int head = nh * 8 + (lane & 3) * 2 + i;
                    if (head >= p.G)
                        continue;
                    float *to = p.scores +
                                (static_cast<size_t>(x.beta) * p.h + static_cast<size_t>(x.j) * p.G + head) *
                                    p.score_stride + static_cast<size_t>(blk) * T + half + (lane >> 2);
#pragma unroll
                    for (int n = 0; n < M; ++n) {   // (rows of scores are whole tiles)
                        to[n * 16] = sc[n][nh][i];
                        to[n * 16 + 8] = sc[n][nh][2 + i];
                    }
                }
        }
        float alpha[NH][2], mu[NH][2];
        bool raised = false;
#pragma unroll
        for (int nh = 0; nh < NH; ++nh)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float mt = neg_inf();
#pragma unroll
                for (int n = 0; n < M; ++n)
                    mt = fmaxf(mt, fmaxf(sc[n][nh][i], sc[n][nh][2 + i]));
#pragma unroll
                for (int d = 4; d < 32; d <<= 1)
                    mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, d));
                const float mn = fmaxf(m[nh][i], mt);
                alpha[nh][i] = m[nh][i] == mn ? 1.f : fast_exp2(m[nh][i] - mn);
                raised = raised || alpha[nh][i] != 1.f;
                m[nh][i] = mn;
                mu[nh][i] = mn == neg_inf() ? 0.f : mn;
                l[nh][i] *= alpha[nh][i];
            }
        if (__any_sync(0xffffffffu, raised)) {
#pragma unroll
            for (int c = 0; c < D / 16; ++c)
#pragma unroll
                for (int nh = 0; nh < NH; ++nh)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[c][nh][e] *= alpha[nh][e & 1];
        }
        // Weights rounded to bf16 for the product (half a step, 2^-8 of each at most); their sum is not.
        uint32_t pf[M][NH][2];
#pragma unroll
        for (int n = 0; n < M; ++n)
#pragma unroll
            for (int nh = 0; nh < NH; ++nh) {
                float w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[e] = fast_exp2(sc[n][nh][e] - mu[nh][e & 1]);
                    l[nh][e & 1] += w[e];
                }
                pf[n][nh][0] = movmatrix_trans(pack_bf16x2(w[0], w[1]));
                pf[n][nh][1] = movmatrix_trans(pack_bf16x2(w[2], w[3]));
            }
#pragma unroll
        for (int n = 0; n < M; ++n)
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                uint32_t a[4];
                ldsm_x4_trans(vb + swz<T>(half + n * 16 + (mi >> 1) * 8 + mr, c * 2 + (mi & 1)), a[0], a[1], a[2],
                              a[3]);
#pragma unroll
                for (int nh = 0; nh < NH; ++nh)
                    mma_bf16_16816(o[c][nh], a, pf[n][nh][0], pf[n][nh][1]);
            }
        __syncwarp();
        if (lane == 0)
            mbar_arrive(bar_empty + 8 * s);
    }
    // The warps' sums meet in the ring (every tile has been read: a consumer takes each).
    const int tid = threadIdx.x;
    float *s_ml = reinterpret_cast<float *>(smem + PL::kML);
#pragma unroll
    for (int nh = 0; nh < NH; ++nh)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1)
                l[nh][i] += __shfl_xor_sync(0xffffffffu, l[nh][i], d);
            if (lane < 4) {
                s_ml[warp * 32 + nh * 8 + lane * 2 + i] = m[nh][i];
                s_ml[warp * 32 + 16 + nh * 8 + lane * 2 + i] = l[nh][i];
            }
        }
    consumer_bar_sync<kWarps>();
    if (tid == 0)
        flag[2] = flag[0];   // (the producer may still give up: one answer for all)
    float *s_o = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int nh = 0; nh < NH; ++nh)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int head = nh * 8 + (lane & 3) * 2 + i;
            if (head < x.rows) {
                float *to = s_o + (warp * 16 + head) * PL::kRow + (lane >> 2);
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    to[c * 16] = o[c][nh][i];
                    to[c * 16 + 8] = o[c][nh][2 + i];
                }
            }
        }
    consumer_bar_sync<kWarps>();
    if (flag[2])
        return;
    if (early && (!p.defer || blockIdx.x == gridDim.x - 1))
        grid_dependency_wait();   // (deferred merge: one CTA, so that this grid ends behind the prefix's)
    const int n_pre = prefix_records<kMode>(p, x.beta);
    const bool defer = kMode == kPieceWeights || group || p.defer;
    const bool whole = !defer && x.count == 1 && n_pre == 0;
    size_t rec = blockIdx.x;
    if constexpr (kMode == kPieceGroups)
        rec -= static_cast<unsigned>(p.n_units);   // (of a unit not used)
    __nv_bfloat16 *ob =
        p.out + (static_cast<size_t>(q_row_of<kMode>(p, x.beta)) * p.h + static_cast<size_t>(x.j) * p.G) * D;
    for (int i = tid * 4; i < x.rows * D; i += kWarps * 32 * 4) {
        const int row = i / D, ch = i - row * D;
        float mx = neg_inf();
#pragma unroll
        for (int w = 0; w < kWarps; ++w)
            mx = fmaxf(mx, s_ml[w * 32 + row]);
        float tot = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float mw = s_ml[w * 32 + row], lw = s_ml[w * 32 + 16 + row];
            // (without a maximum the sum is 0, which has no say, or NaN, which has)
            const float f = mw == neg_inf() ? (lw == 0.f ? 0.f : 1.f) : fast_exp2(mw - mx);
            if (f != 0.f) {
                const float4 v = *reinterpret_cast<const float4 *>(s_o + (w * 16 + row) * PL::kRow + ch);
                tot = fmaf(f, lw, tot);
                acc.x = fmaf(f, v.x, acc.x);
                acc.y = fmaf(f, v.y, acc.y);
                acc.z = fmaf(f, v.z, acc.z);
                acc.w = fmaf(f, v.w, acc.w);
            }
        }
        const float inv = tot == 0.f ? 0.f : 1.f / tot;
        acc.x *= inv;
        acc.y *= inv;
        acc.z *= inv;
        acc.w *= inv;
        if (whole) {
            uint2 w2;
            w2.x = pack_bf16x2(acc.x, acc.y);
            w2.y = pack_bf16x2(acc.z, acc.w);
            *reinterpret_cast<uint2 *>(ob + i) = w2;
        } else {
            float *to_o = p.part_o, *to_lse = p.part_lse;
            size_t to = rec * p.G + row;
            if (group && x.unit) {   // the records of the rows' places
                const int s = row / p.G;
                to_o = const_cast<float *>(p.pre_o);
                to_lse = const_cast<float *>(p.pre_lse);
                to = ((static_cast<size_t>(x.place + s) * p.g + x.j) * p.pre_chunks + x.chunk) * p.G + row - s * p.G;
            }
            *reinterpret_cast<float4 *>(to_o + to * D + ch) = acc;
            if (ch == 0)
                to_lse[to] = tot == 0.f ? neg_inf() : mx + log2f(tot);
        }
    }
    if (whole || defer)
        return;
    if (x.count > 1) {
        __threadfence();
        consumer_bar_sync<kWarps>();
        if (tid == 0)
            flag[1] = static_cast<int>(atomic_add_acq_rel_gpu(&p.counters[x.seg], 1u));
        consumer_bar_sync<kWarps>();
        if (flag[1] != x.count - 1)
            return;
        if (tid == 0)
            p.counters[x.seg] = 0u;
        __threadfence();
    } else {
        __threadfence_block();
        consumer_bar_sync<kWarps>();
    }
    merge_records<D>(p, x, rec - x.index, n_pre, prefix_record<kMode>(p, x.beta, x.j), reinterpret_cast<float *>(smem),
                     tid, kWarps * 32);
}

// The merge of many records by CTAs of their own, 128 floats each: a head of 128 channels or two of 64.  The
// warps take the records in turn, 128 floats a warp and record, eight at a time on the way, and add up in the
// warps' order.  Bound by the records' bytes, in L2, and three round trips to it.  For few records a CTA a segment
// (merge_records): 1024 segments of 6 records of 4 heads of 128 6.4 us, 25 with four of these CTAs each; one segment
// of 152 records of 12 heads of 64 3 us, 23 with one CTA.
constexpr int kWideRecords = 16;
constexpr int kMergeThreads = 256;
template <int D>
struct MergeShared {
    static constexpr int kRows = 128 / D;   // heads of a CTA; the last one may be past the group
    float inv[kRows];
    float4 sum[kMergeThreads / 32][32];
};
template <int D>
__device__ void merge_rows(MergeShared<D> &sh, const PieceBase &p, const Piece &x, size_t own0, int n_pre, size_t pre0,
                           int part, float *s_w)
{
    constexpr int R = MergeShared<D>::kRows, W = kMergeThreads / 32, U = 8;
    const int G = p.G, n = x.count + n_pre, tid = static_cast<int>(threadIdx.x), warp = tid >> 5, lane = tid & 31;
    auto lse_of = [&](int k, int head) {
        return k < x.count ? __ldcg(p.part_lse + (own0 + k) * G + head)
                           : __ldcg(p.pre_lse + (pre0 + (k - x.count)) * G + head);
    };
    for (int i = tid; i < n * R; i += kMergeThreads) {
        const int head = part * R + i % R;
        s_w[i] = head < G ? lse_of(i / R, head) : neg_inf();
    }
    __syncthreads();
    if (warp < R) {
        float mx = neg_inf(), tot = 0.f;
        for (int k = lane; k < n; k += 32)
            mx = fmaxf(mx, s_w[k * R + warp]);
        for (int d = 16; d > 0; d >>= 1)
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
        for (int k = lane; k < n; k += 32) {
            const float lse = s_w[k * R + warp];
            const float w = lse == neg_inf() ? 0.f : fast_exp2(lse - mx);   // (a NaN goes on)
            s_w[k * R + warp] = w;
            tot += w;
        }
        for (int d = 16; d > 0; d >>= 1)
            tot += __shfl_xor_sync(0xffffffffu, tot, d);
        if (lane == 0)
            sh.inv[warp] = tot == 0.f ? 0.f : 1.f / tot;
    }
    __syncthreads();
    const int r = lane * 4 / D, head = part * R + r;
    const bool live = head < G;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k0 = warp; live && k0 < n; k0 += U * W) {
        float4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + u * W;
            const float *rec = k < x.count ? p.part_o + (own0 + k) * G * D : p.pre_o + (pre0 + (k - x.count)) * G * D;
            v[u] = k < n ? __ldcg(reinterpret_cast<const float4 *>(rec + part * 128) + lane)
                         : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + u * W;
            const float w = k < n ? s_w[k * R + r] : 0.f;
            if (w != 0.f) {
                acc.x = fmaf(w, v[u].x, acc.x);
                acc.y = fmaf(w, v[u].y, acc.y);
                acc.z = fmaf(w, v[u].z, acc.z);
                acc.w = fmaf(w, v[u].w, acc.w);
            }
        }
    }
    sh.sum[warp][lane] = acc;
    __syncthreads();
    if (warp == 0 && live) {
#pragma unroll
        for (int w = 1; w < W; ++w) {
            const float4 v = sh.sum[w][lane];
            acc.x += v.x;
            acc.y += v.y;
            acc.z += v.z;
            acc.w += v.w;
        }
        const float inv = sh.inv[r];
        uint2 w2;
        w2.x = pack_bf16x2(acc.x * inv, acc.y * inv);
        w2.y = pack_bf16x2(acc.z * inv, acc.w * inv);
        *reinterpret_cast<uint2 *>(p.out + (static_cast<size_t>(x.out_row) * p.h + static_cast<size_t>(x.j) * G) * D +
                                   part * 128 + lane * 4) = w2;
    }
}

// The segment of KV head k % g of the (k / g)-th row as they are laid out, whose records begin at *own0.
template <int kMode>
__device__ __forceinline__ Piece segment_of(const PieceArgs<kMode> &p, int k, size_t *own0)
{
    Piece x;
    const int i = k / p.g;
    x.beta = row_at(p, i);
    x.j = k - i * p.g;
    x.seg = x.beta * p.g + x.j;
    x.L = p.seq_len[x.beta];
    x.count = (piece_tiles<kMode>(p, x.beta) + p.tiles - 1) / p.tiles;
    x.out_row = q_row_of<kMode>(p, x.beta);
    *own0 = static_cast<size_t>(p.first[i]) + static_cast<size_t>(x.j) * x.count;
    return x;
}

template <int D, int kMode, bool kWide>
__global__ void __launch_bounds__(kWide ? kMergeThreads : 128) merge_kernel(const __grid_constant__ PieceArgs<kMode> p)
{
    extern __shared__ float s_w[];
    const int parts = kWide ? (p.G * D + 127) / 128 : 1, seg = static_cast<int>(blockIdx.x) / parts;
    size_t own0;
    const Piece x = segment_of<kMode>(p, seg, &own0);
    const int n_pre = prefix_records<kMode>(p, x.beta);
    const size_t pre0 = prefix_record<kMode>(p, x.beta, x.j);
    grid_dependency_wait();
    grid_dependents_launch();
    if constexpr (kWide) {
        __shared__ MergeShared<D> sh;
        merge_rows<D>(sh, p, x, own0, n_pre, pre0, static_cast<int>(blockIdx.x) % parts, s_w);
    } else {
        merge_records<D>(p, x, own0, n_pre, pre0, s_w, static_cast<int>(threadIdx.x), 128);
    }
}

// --------------------------------------------------------------------------------------------------
// kPieceWeights: what each position got
// --------------------------------------------------------------------------------------------------

// A segment's first CTAs merge its records into out, the others take a chunk of its positions each.  Bound by the
// scores' and weights' bytes, 4 G + 8 a position of a KV head (the scores from L2 where they fit): 32 sequences of
// 8192 positions, 8 KV heads of 4 heads each, 13 us beside the pieces.
constexpr int kWeightThreads = 256;
template <int D>
__global__ void __launch_bounds__(kWeightThreads, 4)
    weights_kernel(const __grid_constant__ PieceBase p, const __grid_constant__ WeightsParams w)
{
    __shared__ float s_lse[16];
    extern __shared__ float s_w[];
    grid_dependency_wait();
    grid_dependents_launch();
    static_assert(kWeightThreads == kMergeThreads, "one size of CTA");
    __shared__ MergeShared<D> sh;
    const int seg = static_cast<int>(blockIdx.x) / w.ctas, tid = static_cast<int>(threadIdx.x);
    const int parts = w.merge_ctas;
    const int part = static_cast<int>(blockIdx.x) - seg * w.ctas - parts;   // chunk of positions
    size_t rec0;
    const Piece x = segment_of<kPieceWeights>(p, seg, &rec0);
    const int G = p.G;
    if (part < 0) {
        if (w.wide)
            merge_rows<D>(sh, p, x, rec0, 0, 0, part + parts, s_w);
        else
            merge_records<D>(p, x, rec0, 0, 0, s_w, tid, kWeightThreads);
        return;
    }
    const int u0 = part * w.chunk, u1 = min(u0 + w.chunk, w.max_seq);
    const size_t row = static_cast<size_t>(x.seg) * w.max_seq;
    const float *sc = p.scores + (static_cast<size_t>(x.beta) * p.h + static_cast<size_t>(x.j) * G) * p.score_stride;
    constexpr int U = 4, B = 4;   // positions of a thread, and heads, at a time
    float s[B][U], before[U];
    auto fetch = [&](int v, int i0) {
#pragma unroll
        for (int i = 0; i < B; ++i)
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int u = v + k * kWeightThreads;
                s[i][k] = i0 + i < G && u < min(x.L, u1) ? __ldcg(sc + (i0 + i) * p.score_stride + u) : neg_inf();
            }
    };
    auto fetch_before = [&](int v) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int u = v + k * kWeightThreads;
            before[k] = w.weights_in != nullptr && u < u1 ? w.weights_in[row + u] : 0.f;
        }
    };
    fetch(u0 + tid, 0);   // (on the way while the sums are added up)
    fetch_before(u0 + tid);
    if (u0 < x.L) {
        // log2 of every head's sum, from the records: a warp a head
        for (int i = tid >> 5; i < G; i += kWeightThreads / 32) {
            const int lane = tid & 31;
            float mx = neg_inf();
            for (int k = lane; k < x.count; k += 32)
                mx = fmaxf(mx, __ldcg(p.part_lse + (rec0 + k) * G + i));
            for (int d = 16; d > 0; d >>= 1)
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
            float tot = 0.f;
            for (int k = lane; k < x.count; k += 32) {
                const float lse = __ldcg(p.part_lse + (rec0 + k) * G + i);
                tot += lse == neg_inf() ? 0.f : exp2f(lse - mx);
            }
            for (int d = 16; d > 0; d >>= 1)
                tot += __shfl_xor_sync(0xffffffffu, tot, d);
            if (lane == 0)
                s_lse[i] = tot == 0.f ? 0.f : mx + log2f(tot);   // (scores that are all -inf: no weight)
        }
        __syncthreads();
    }
    for (int v = u0 + tid; v < u1; v += U * kWeightThreads) {
        if (v != u0 + tid) {
            fetch(v, 0);
            fetch_before(v);
        }
        float a[U];
#pragma unroll
        for (int k = 0; k < U; ++k)
            a[k] = 0.f;
        for (int i0 = 0; v < x.L && i0 < G; i0 += B) {
            if (i0 > 0)
                fetch(v, i0);
#pragma unroll
            for (int i = 0; i < B; ++i) {
                if (i0 + i >= G)
                    break;
                const float lse = s_lse[i0 + i];
#pragma unroll
                for (int k = 0; k < U; ++k)
                    a[k] += fast_exp2(s[i][k] - lse);
            }
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int u = v + k * kWeightThreads;
            if (u < u1)
                w.weights_out[row + u] = before[k] + (u < x.L ? a[k] : 0.f);   // (a NaN ends with its sequence)
        }
    }
}

template <int D, int NH>
const void *piece_fn(int mode)
{
    return mode == kPieceSuffix   ? reinterpret_cast<const void *>(&piece_kernel<D, kPieceSuffix, NH>)
           : mode == kPieceBlocks ? reinterpret_cast<const void *>(&piece_kernel<D, kPieceBlocks, NH>)
           : mode == kPieceJoined ? reinterpret_cast<const void *>(&piece_kernel<D, kPieceJoined, NH>)
           : mode == kPieceGroups ? reinterpret_cast<const void *>(&piece_kernel<D, kPieceGroups, 2>)
                                  : reinterpret_cast<const void *>(&piece_kernel<D, kPieceWeights, NH>);
}
const void *piece_fn(int head_dim, int G, int mode)
{
    if (G <= 8)
        return head_dim == 64 ? piece_fn<64, 1>(mode) : piece_fn<128, 1>(mode);
    return head_dim == 64 ? piece_fn<64, 2>(mode) : piece_fn<128, 2>(mode);
}

int piece_threads(int head_dim) { return head_dim == 64 ? PiecePlan<64>::kThreads : PiecePlan<128>::kThreads; }
size_t piece_smem(int head_dim) { return head_dim == 64 ? PiecePlan<64>::kBytes : PiecePlan<128>::kBytes; }

// The mode's part of the parameters (PieceArgs).
void *args_of(int mode, const PieceParams &p)
{
    if (mode == kPieceGroups)
        return const_cast<PieceParams *>(&p);
    if (mode == kPieceSuffix || mode == kPieceJoined)
        return const_cast<PiecePrefix *>(static_cast<const PiecePrefix *>(&p));
    return const_cast<PieceBase *>(static_cast<const PieceBase *>(&p));
}

cudaError_t launch_pdl(const void *fn, dim3 grid, int threads, size_t smem, cudaStream_t stream, void **args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelExC(&cfg, fn, args);
}

}  // namespace

int piece_stages(int head_dim) { return head_dim == 64 ? PiecePlan<64>::kStages : PiecePlan<128>::kStages; }

int piece_max_records(int head_dim, int G)
{
    return (head_dim == 64 ? max_records<64>(G) : max_records<128>(G)) - 1;
}

cudaError_t prepare_pieces(int head_dim, int G, int mode, int *ctas_per_sm)
{
    const void *fn = piece_fn(head_dim, G, mode);
    cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         static_cast<int>(piece_smem(head_dim)));
    if (e == cudaSuccess)
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(ctas_per_sm, fn, piece_threads(head_dim),
                                                          piece_smem(head_dim));
    return e;
}

cudaError_t launch_pieces(int head_dim, int mode, const CUtensorMap *tmap, const CUtensorMap *tmap_prefix,
                          const PieceParams &p, cudaStream_t stream)
{
    void *args[] = {const_cast<CUtensorMap *>(tmap), const_cast<CUtensorMap *>(tmap_prefix),
                    args_of(mode, p)};
    const int ctas = p.first[p.n] + (mode == kPieceGroups ? p.n_units : 0);
    return launch_pdl(piece_fn(head_dim, p.G, mode), dim3(static_cast<unsigned>(ctas)), piece_threads(head_dim),
                      piece_smem(head_dim), stream, args);
}

// Room for the merge's weights.
size_t merge_smem(int head_dim, int G, int most)
{
    return sizeof(float) * (most > kWideRecords ? static_cast<size_t>(most) * (128 / head_dim)
                                                : (static_cast<size_t>(most) + 1) * G);
}

template <int D, int kMode>
const void *merge_fn(bool wide)
{
    return wide ? reinterpret_cast<const void *>(&merge_kernel<D, kMode, true>)
                : reinterpret_cast<const void *>(&merge_kernel<D, kMode, false>);
}
template <int D>
const void *merge_fn(int mode, bool wide)
{
    return mode == kPieceBlocks   ? merge_fn<D, kPieceBlocks>(wide)
           : mode == kPieceJoined ? merge_fn<D, kPieceJoined>(wide)
           : mode == kPieceGroups ? merge_fn<D, kPieceGroups>(wide)
                                  : merge_fn<D, kPieceSuffix>(wide);
}

cudaError_t launch_merge_pieces(int head_dim, int mode, const PieceParams &p, int most, cudaStream_t stream)
{
    const bool wide = most > kWideRecords;
    const void *fn = head_dim == 64 ? merge_fn<64>(mode, wide) : merge_fn<128>(mode, wide);
    void *args[] = {args_of(mode, p)};
    const unsigned ctas = wide ? static_cast<unsigned>((p.G * head_dim + 127) / 128) : 1u;
    return launch_pdl(fn, dim3(ctas * static_cast<unsigned>(p.n) * p.g), wide ? kMergeThreads : 128,
                      merge_smem(head_dim, p.G, most), stream, args);
}

void plan_weights(int head_dim, int G, int most, WeightsParams *w)
{
    w->wide = most > kWideRecords ? 1 : 0;
    w->merge_ctas = w->wide ? (G * head_dim + 127) / 128 : 1;
}

cudaError_t launch_weights(int head_dim, const PieceParams &p, const WeightsParams &w, int most,
                           cudaStream_t stream)
{
    const size_t smem = merge_smem(head_dim, p.G, most);
    void *args[] = {args_of(kPieceWeights, p), const_cast<WeightsParams *>(&w)};
    return launch_pdl(head_dim == 64 ? reinterpret_cast<const void *>(&weights_kernel<64>)
                                     : reinterpret_cast<const void *>(&weights_kernel<128>),
                      dim3(static_cast<unsigned>(w.ctas) * p.b * p.g), kWeightThreads, smem, stream, args);
}

}  // namespace mlkv
