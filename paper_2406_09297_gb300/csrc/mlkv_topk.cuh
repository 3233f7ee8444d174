// The n largest of a list of 32-bit keys that a thread-block cluster holds, in the order of the list.  Of equal
// keys the first ones are taken, so that the selection does not depend on how the list is split.  Used by
// the block selection and the eviction.  Internal.
//
// The last key taken is found by histograms of 1024 equal intervals between the least and the largest key, then
// of the interval that holds it, and so on until all of an interval's keys are taken or it is one key wide: two
// rounds for weights or scores as they come, at most four.  (Digits of eight bits, from the top: the keys are floats
// whose upper digit is an exponent that most share, and four rounds are always four: eviction from 16 sequences of
// up to 16,384 positions, 8 KV heads, 26.4 us a selection.)
#pragma once

#include <cooperative_groups.h>

#include "mlkv_device.cuh"

namespace mlkv {
namespace {

constexpr int kTopkBins = 1024;
constexpr unsigned kTopkCluster = 8;   // CTAs of a cluster, at most

template <int NT>
struct TopkShared {
    unsigned hist[2][kTopkBins];   // of this CTA's keys; the rounds take turns
    unsigned warp[NT / 32];
    unsigned lo, hi;               // least and largest key of this CTA
    unsigned bin, above, inside;   // interval of the last key taken; keys above it, and in it
    unsigned gt, eq;               // this CTA's keys above the last one taken, and equal to it
    unsigned warp_gt[NT / 32], warp_eq[NT / 32];
};

// CTA `rank` of a cluster of `size` holds keys key(0) .. key(n - 1), whose least and largest are lo and hi in
// all threads (0xffffffff and 0 of none); the cluster (size 1: this CTA alone, whatever its cluster) holds at least
// `want` >= 1 keys.  Calls put(place, i) for every one of its keys among the `want` largest, place its rank in the
// list's order among those.  All NT >= 256 threads of all the cluster's CTAs call it, behind a barrier for the keys.
template <int NT, typename Key, typename Put>
__device__ void cluster_topk(TopkShared<NT> &sh, unsigned size, unsigned rank, int n, unsigned lo, unsigned hi,
                             unsigned want, const Key &key, const Put &put)
{
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = static_cast<int>(threadIdx.x), lane = tid & 31, warp = tid >> 5;
    constexpr int W = NT / 32;
    auto sync = [&] {
        if (size > 1)
            cluster.sync();
        else
            __syncthreads();
    };
    for (int b = tid; b < kTopkBins; b += NT)
        sh.hist[0][b] = 0;
    if (size > 1) {
        if (tid == 0) {
            sh.lo = lo;
            sh.hi = hi;
        }
        cluster.sync();
#pragma unroll
        for (unsigned c = 0; c < kTopkCluster; ++c)
            if (c < size) {
                lo = min(lo, *cluster.map_shared_rank(&sh.lo, c));
                hi = max(hi, *cluster.map_shared_rank(&sh.hi, c));
            }
    } else {
        __syncthreads();
    }
    unsigned left = want;   // keys still to take of [lo, hi]
    bool all = false;       // every key of [lo, hi] is taken
    for (int round = 0; round < 4 && !all && lo != hi; ++round) {   // (widths 2^32, 2^22, 2^12, 4)
        unsigned *hist = sh.hist[round & 1];
        const int s = max(0, 22 - __clz(static_cast<int>(hi - lo)));   // (hi - lo) >> s below 1024
        // (keys that equal lo are counted apart: where many weights are the same, they are mostly the least)
        unsigned at_lo = 0;
        for (int i = tid; i < n; i += NT) {
            const unsigned k = key(i);
            at_lo += k == lo;
            if (k > lo && k <= hi)
                atomicAdd(&hist[(k - lo) >> s], 1u);
        }
        at_lo = __reduce_add_sync(0xffffffffu, at_lo);
        if (lane == 0 && at_lo > 0)
            atomicAdd(&hist[0], at_lo);
        sync();
        // the cluster's counts from the top: thread t takes the kPer intervals below kTopkBins - kPer t
        constexpr int kPer = kTopkBins >= NT ? kTopkBins / NT : 1;
        unsigned mine[kPer], total = 0;
        const bool has = tid * kPer < kTopkBins;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            mine[k] = 0;
            if (has) {
                const int b = kTopkBins - 1 - tid * kPer - k;
                if (size == 1) {
                    mine[k] = hist[b];
                } else {
                    unsigned v[kTopkCluster];   // (all on the way at once)
#pragma unroll
                    for (unsigned c = 0; c < kTopkCluster; ++c)
                        v[c] = c < size ? *cluster.map_shared_rank(&hist[b], c) : 0u;
#pragma unroll
                    for (unsigned c = 0; c < kTopkCluster; ++c)
                        mine[k] += v[c];
                }
            }
            total += mine[k];
        }
        for (int b = tid; b < kTopkBins; b += NT)
            sh.hist[(round + 1) & 1][b] = 0;   // (read last before the sync above)
        unsigned up = total;
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned o = __shfl_up_sync(0xffffffffu, up, d);
            if (lane >= d)
                up += o;
        }
        if (lane == 31)
            sh.warp[warp] = up;
        __syncthreads();
        unsigned before = lane < W && lane < warp ? sh.warp[lane] : 0;
        before = __reduce_add_sync(0xffffffffu, before);
        unsigned above = before + up - total;
        if (above < left && left <= before + up) {
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                if (above < left && left <= above + mine[k]) {
                    sh.bin = static_cast<unsigned>(kTopkBins - 1 - tid * kPer - k);
                    sh.above = above;
                    sh.inside = mine[k];
                }
                above += mine[k];
            }
        }
        __syncthreads();
        left -= sh.above;
        all = sh.inside == left;
        lo += sh.bin << s;
        hi = lo + min(hi - lo, (1u << s) - 1u);   // (the interval's end may lie past 2^32)
    }
    // Keys above `top` are taken, and the first `left` that equal it (none where whole intervals are taken).  Each
    // warp has a run of the CTA's keys.
    const unsigned top = all ? lo - 1u : lo;   // (all of [0, hi]: every key, and above 0xffffffff is none)
    const bool every = all && lo == 0u;
    if (all)
        left = 0;
    const int run = ((n + W - 1) / W + 31) & ~31;
    const int i0 = min(n, warp * run), i1 = min(n, i0 + run);
    unsigned gt = 0, eq = 0;
    for (int i = i0 + lane; i < i1; i += 32) {
        const unsigned k = key(i);
        gt += every || k > top;
        eq += !all && k == top;
    }
    gt = __reduce_add_sync(0xffffffffu, gt);
    eq = __reduce_add_sync(0xffffffffu, eq);
    if (lane == 0) {
        sh.warp_gt[warp] = gt;
        sh.warp_eq[warp] = eq;
    }
    __syncthreads();
    const unsigned a = lane < W ? sh.warp_gt[lane] : 0u, b = lane < W ? sh.warp_eq[lane] : 0u;
    unsigned gt0 = __reduce_add_sync(0xffffffffu, lane < warp ? a : 0u);   // before this warp's run
    unsigned eq0 = __reduce_add_sync(0xffffffffu, lane < warp ? b : 0u);
    if (size > 1) {
        const unsigned ga = __reduce_add_sync(0xffffffffu, a), ea = __reduce_add_sync(0xffffffffu, b);
        if (tid == 0) {
            sh.gt = ga;
            sh.eq = ea;
        }
        cluster.sync();
#pragma unroll
        for (unsigned c = 0; c < kTopkCluster; ++c)
            if (c < rank) {
                gt0 += *cluster.map_shared_rank(&sh.gt, c);
                eq0 += *cluster.map_shared_rank(&sh.eq, c);
            }
    }
    for (int i = i0; i < i1; i += 32) {
        const bool in = i + lane < i1;
        const unsigned k = in ? key(i + lane) : 0u;
        const bool is_gt = in && (every || k > top), is_eq = in && !all && k == top;
        const unsigned bg = __ballot_sync(0xffffffffu, is_gt), be = __ballot_sync(0xffffffffu, is_eq);
        const unsigned below = (1u << lane) - 1u;
        const unsigned g = gt0 + __popc(bg & below), e = eq0 + __popc(be & below);
        if (is_gt || (is_eq && e < left))
            put(g + min(e, left), i + lane);
        gt0 += __popc(bg);
        eq0 += __popc(be);
    }
    if (size > 1)
        cluster.sync();   // no CTA leaves while its counts are read
}

// The least and the largest over the CTA's threads; s: room for 2 * NT / 32 numbers.
template <int NT>
__device__ __forceinline__ void block_min_max(unsigned &lo, unsigned &hi, unsigned *s)
{
    const int lane = static_cast<int>(threadIdx.x) & 31, warp = static_cast<int>(threadIdx.x) >> 5;
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) {
        s[warp] = lo;
        s[NT / 32 + warp] = hi;
    }
    __syncthreads();
    lo = __reduce_min_sync(0xffffffffu, lane < NT / 32 ? s[lane] : 0xffffffffu);
    hi = __reduce_max_sync(0xffffffffu, lane < NT / 32 ? s[NT / 32 + lane] : 0u);
}

}  // namespace
}  // namespace mlkv
