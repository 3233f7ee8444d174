// The n largest of a list of 32-bit keys that a thread-block cluster holds, in the order of the list: a radix
// select of four digits of eight bits.  Of equal keys the first ones are taken, so that the selection does not
// depend on how the list is split.  Used by the block selection and the eviction.  Internal.
#pragma once

#include <cooperative_groups.h>

#include "mlkv_device.cuh"

namespace mlkv {
namespace {

constexpr int kTopkThreads = 512;

struct TopkShared {
    unsigned hist[2][256];   // of this CTA's keys, by digit; the digits take turns
    unsigned sum[256];       // of the cluster's, from this digit up
    unsigned digit, above;   // the digit of the last key taken; keys above it
    unsigned gt, eq;         // this CTA's keys above the last one taken, and equal to it
    unsigned warp_gt[kTopkThreads / 32], warp_eq[kTopkThreads / 32];
};

// CTA `rank` of `size` holds keys key(0) .. key(n - 1), the list's first_index and following ones; the cluster
// holds at least `want` >= 1 keys.  Calls put(place, i) for every one of its keys among the `want` largest, place
// its rank in the list's order among those.  All threads of the cluster call it.
template <typename Key, typename Put>
__device__ void cluster_topk(TopkShared &sh, int n, unsigned want, const Key &key, const Put &put)
{
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const unsigned size = cluster.num_blocks(), rank = cluster.block_rank();
    const int tid = static_cast<int>(threadIdx.x), lane = tid & 31, warp = tid >> 5;
    constexpr int W = kTopkThreads / 32;
    auto sync = [&] {
        if (size > 1)
            cluster.sync();
        else
            __syncthreads();
    };
    unsigned prefix = 0, left = want;   // the last taken key's upper digits; keys still to take below
    for (int d = 3; d >= 0; --d) {
        unsigned *hist = sh.hist[d & 1];
        if (tid < 256)
            hist[tid] = 0;
        __syncthreads();
        const unsigned high = d == 3 ? 0u : ~0u << (8 * (d + 1));
        for (int base = warp * 32; base < n; base += kTopkThreads) {
            const unsigned k = base + lane < n ? key(base + lane) : 0u;
            const unsigned b = (k >> (8 * d)) & 255u;
            const bool in = base + lane < n && (k & high) == prefix;
            // (many keys share a digit: one addition for the lanes that agree with the warp's first)
            const unsigned live = __ballot_sync(0xffffffffu, in);
            if (live == 0)
                continue;
            const int lead = __ffs(static_cast<int>(live)) - 1;
            const unsigned b0 = __shfl_sync(0xffffffffu, b, lead);
            const unsigned same = __ballot_sync(0xffffffffu, in && b == b0);
            if (in && b != b0)
                atomicAdd(&hist[b], 1u);
            else if (lane == lead)
                atomicAdd(&hist[b0], static_cast<unsigned>(__popc(same)));
        }
        sync();
        if (tid < 256) {
            unsigned t = 0;
            for (unsigned c = 0; c < size; ++c)
                t += *cluster.map_shared_rank(&hist[tid], c);
            sh.sum[tid] = t;
        }
        __syncthreads();
        if (warp == 0) {
            // from the top: lane i takes digits 255 - 8 i downwards
            unsigned mine = 0;
            for (int k = 0; k < 8; ++k)
                mine += sh.sum[255 - 8 * lane - k];
            unsigned up = mine;   // keys of this lane's digits and those above
            for (int s = 1; s < 32; s <<= 1) {
                const unsigned o = __shfl_up_sync(0xffffffffu, up, s);
                if (lane >= s)
                    up += o;
            }
            unsigned above = up - mine;
            if (above < left && left <= up) {
                for (int k = 0; k < 8; ++k) {
                    const unsigned c = sh.sum[255 - 8 * lane - k];
                    if (above + c >= left) {
                        sh.digit = 255u - 8u * lane - k;
                        sh.above = above;
                        break;
                    }
                    above += c;
                }
            }
        }
        __syncthreads();
        prefix |= sh.digit << (8 * d);
        left -= sh.above;
    }
    // Keys above `prefix` are taken, and the first `left` that equal it.  Each warp has a run of the CTA's keys.
    const int run = ((n + W - 1) / W + 31) & ~31;
    const int i0 = min(n, warp * run), i1 = min(n, i0 + run);
    unsigned gt = 0, eq = 0;
    for (int i = i0 + lane; i < i1; i += 32) {
        const unsigned k = key(i);
        gt += k > prefix;
        eq += k == prefix;
    }
    for (int s = 16; s > 0; s >>= 1) {
        gt += __shfl_xor_sync(0xffffffffu, gt, s);
        eq += __shfl_xor_sync(0xffffffffu, eq, s);
    }
    if (lane == 0) {
        sh.warp_gt[warp] = gt;
        sh.warp_eq[warp] = eq;
    }
    __syncthreads();
    if (tid == 0) {
        unsigned a = 0, b = 0;
        for (int w = 0; w < W; ++w) {
            a += sh.warp_gt[w];
            b += sh.warp_eq[w];
        }
        sh.gt = a;
        sh.eq = b;
    }
    sync();
    unsigned gt0 = 0, eq0 = 0;   // before this warp's run
    for (unsigned c = 0; c < rank; ++c) {
        gt0 += *cluster.map_shared_rank(&sh.gt, c);
        eq0 += *cluster.map_shared_rank(&sh.eq, c);
    }
    for (int w = 0; w < warp; ++w) {
        gt0 += sh.warp_gt[w];
        eq0 += sh.warp_eq[w];
    }
    for (int i = i0; i < i1; i += 32) {
        const unsigned k = i + lane < i1 ? key(i + lane) : 0u;
        const bool is_gt = i + lane < i1 && k > prefix, is_eq = i + lane < i1 && k == prefix;
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

}  // namespace
}  // namespace mlkv
