// Eviction from a KV cache by accumulated attention weight, for GB300: of every (sequence, KV head) the
// `recent` newest positions stay and, of the others, those of the largest weights, `keep` in all, of equal
// weights the earlier ones; keys, values and weights of what stays move together, in order.
//
// keep_kernel selects: a cluster a segment, over its weights as ordered keys (cluster_topk), whose result is the list of
// kept positions; what stays of short segments it moves as well, in rounds.  Else move_kernel moves: a unit is a run of
// rows of a segment, which a CTA loads whole before it stores it.  In place, row m takes position kept[m] >= m, so a unit overwrites positions
// that only units before it, and it itself, still have to read: it stores after those have set their flags.
// Units are handed out by a counter in rising order within a segment, so that what a unit waits for has been
// handed out before it and is running: no wait depends on a CTA that has not started.
// Bound by the bytes of what stays, read and written once, and by the selection's latency: 4096 positions kept of each of
// 16 uneven sequences of up to 16,384, 8 KV heads of 128, 13.2 us to select, 72 us to move 423 MB into another cache,
// 5.9 TB/s. In place, where units wait for those whose rows they overwrite, 106 us, 4.0 TB/s.
#include "mlkv_device.cuh"
#include "mlkv_long.h"
#include "mlkv_topk.cuh"

namespace mlkv {
namespace {

constexpr size_t kKeepSmem = 128 * 1024;   // keys of a CTA that fit in shared memory
constexpr int kMaxCluster = kTopkCluster;

// Ordered as the weights, both zeros alike, NaN above infinity.
__device__ __forceinline__ unsigned weight_key(float w)
{
    const uint32_t u = __float_as_uint(w + 0.f);
    return w != w ? 0xfffffffeu : (u >> 31) ? ~u : u | 0x80000000u;
}

constexpr int kKeepThreads = 1024, kKeepFew = 256;   // of a CTA; of one among many

constexpr int kKeepVecs = 4;   // 16-byte vectors of a thread and round, where it moves as well

// D: 0, or the head_dim of rows that it moves as well.
template <int D, int NT>
__global__ void __launch_bounds__(NT, kKeepThreads / NT) keep_kernel(const __grid_constant__ EvictParams p)
{
    namespace cg = cooperative_groups;
    __shared__ TopkShared<NT> sh;
    __shared__ unsigned s_mm[2 * NT / 32];
    extern __shared__ unsigned s_key[];
    cg::cluster_group cluster = cg::this_cluster();
    const int size = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int seg = static_cast<int>(blockIdx.x) / size, beta = seg / p.g;
    const int tid = static_cast<int>(threadIdx.x);
    const int L = p.seq_len[beta], keep = p.keep[beta];
    const float *w = p.weights_in + static_cast<size_t>(seg) * p.src_seq;
    int *kept = p.kept + static_cast<size_t>(seg) * p.k_max;
    grid_dependency_wait();
    grid_dependents_launch();
    if constexpr (D == 0) {
        // the flags of this segment's units; the first CTA also resets the counter of units
        for (int i = rank * NT + tid; i < p.units; i += size * NT)
            p.flags[static_cast<size_t>(seg) * p.units + i] = 0u;
        if (blockIdx.x == 0 && tid == 0)
            p.flags[static_cast<size_t>(p.b) * p.g * p.units] = 0u;
    }
    // Everything stays of a shorter sequence, else the newest positions, and the heaviest of the others.
    const int others = L <= keep ? 0 : L - p.recent, want = L <= keep ? 0 : keep - p.recent;
    for (int i = rank * NT + tid; i < min(L, keep) - want; i += size * NT)
        kept[want + i] = others + i;
    if (want > 0) {
        const int per = (others + size - 1) / size;
        const int first = min(others, rank * per), n = min(others, first + per) - first;
        const bool cached = static_cast<size_t>(per) * 4 <= kKeepSmem;
        unsigned least = 0xffffffffu, most = 0u;
        constexpr int U = 8;   // loads in flight
        for (int i0 = tid; i0 < n; i0 += U * NT) {
            float x[U];
    #pragma unroll
            for (int u = 0; u < U; ++u)
                x[u] = i0 + u * NT < n ? __ldcg(w + first + i0 + u * NT) : 0.f;
    #pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u * NT < n) {
                    const unsigned k = weight_key(x[u]);
                    least = min(least, k);
                    most = max(most, k);
                    if (cached)
                        s_key[i0 + u * NT] = k;
                }
        }
        block_min_max<NT>(least, most, s_mm);   // (and the keys are in place)
        cluster_topk<NT>(sh, size, rank, n, least, most, static_cast<unsigned>(want),
                         [&](int i) { return cached ? s_key[i] : weight_key(__ldcg(w + first + i)); },
                         [&](unsigned place, int i) { kept[place] = first + i; });
    }
    if constexpr (D > 0) {
        // Rows in rounds, a run of them a CTA.  In place, row m takes position kept[m] >= m: a round stores over
        // positions that none of the later ones reads, once all of its own have been read.
        constexpr int C = D / 8, R = NT * kKeepVecs / (2 * C);
        auto sync = [&] {
            if (size > 1)
                cluster.sync();
            else
                __syncthreads();
        };
        const int rows = min(L, keep), segments = p.b * p.g;
        float *w_out = p.weights_out + static_cast<size_t>(seg) * p.dst_seq;
        sync();   // the list is there
        for (int m0 = 0; m0 < rows; m0 += size * R) {
            const int at = m0 + rank * R, n_here = min(R, rows - at);   // (none or less at the end)
            uint4 v[kKeepVecs];
            float x = 0.f;
#pragma unroll
            for (int k = 0; k < kKeepVecs; ++k) {
                const int i = k * NT + tid, kv = i / (R * C), row = i % (R * C) / C, c = i % C;   // K's vectors, then V's
                if (row < n_here)
                    v[k] = __ldcs(
                        reinterpret_cast<const uint4 *>(p.src) +
                        ((static_cast<size_t>(kv) * segments + seg) * p.src_seq + __ldcg(kept + at + row)) * C + c);
            }
            if (tid < n_here)
                x = __ldcg(w + __ldcg(kept + at + tid));
            if (p.in_place) {
                __threadfence();   // (the loads have happened, not only been issued)
                sync();
            }
#pragma unroll
            for (int k = 0; k < kKeepVecs; ++k) {
                const int i = k * NT + tid, kv = i / (R * C), row = i % (R * C) / C, c = i % C;
                if (row < n_here)
                    __stcs(reinterpret_cast<uint4 *>(p.dst) +
                               ((static_cast<size_t>(kv) * segments + seg) * p.dst_seq + at + row) * C + c, v[k]);
            }
            if (tid < n_here)
                w_out[at + tid] = x;
        }
        for (int u = rows + rank * NT + tid; u < p.dst_seq; u += size * NT)
            w_out[u] = 0.f;
    }
}

constexpr int kMoveThreads = 256;
constexpr int kUnitVecs = 8;   // 16-byte vectors of a thread and unit

// Rows of a unit: its keys and values are kMoveThreads * kUnitVecs vectors.
template <int D>
__host__ __device__ constexpr int unit_rows() { return kMoveThreads * kUnitVecs / (2 * D / 8); }

__device__ __forceinline__ unsigned ld_acquire(const unsigned *p)
{
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void st_release(unsigned *p, unsigned v)
{
    asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}

template <int D>
__global__ void __launch_bounds__(kMoveThreads) move_kernel(const __grid_constant__ EvictParams p)
{
    constexpr int R = unit_rows<D>(), C = D / 8;
    __shared__ int s_at[R];
    __shared__ unsigned s_unit;
    __shared__ int s_first, s_ok, s_move;
    const int tid = static_cast<int>(threadIdx.x);
    const int segments = p.b * p.g;
    const unsigned total = static_cast<unsigned>(segments) * p.units;
    unsigned *ticket = p.flags + static_cast<size_t>(segments) * p.units;
    grid_dependency_wait();
    grid_dependents_launch();
    for (;;) {
        __syncthreads();
        if (tid == 0)
            s_unit = atomicAdd(ticket, 1u);
        __syncthreads();
        const unsigned unit = s_unit;
        if (unit >= total)
            return;
        // units of one segment in rising order, the segments side by side
        const int r = static_cast<int>(unit / segments), seg = static_cast<int>(unit % segments);
        const int beta = seg / p.g;
        const int L = p.seq_len[beta];
        const int n = min(L, p.keep[beta]);
        unsigned *flags = p.flags + static_cast<size_t>(seg) * p.units;
        const int last = (n + R - 1) / R;   // the segment's units of rows; behind them one for the tail
        if (r > last)
            continue;
        const float *w_in = p.weights_in + static_cast<size_t>(seg) * p.src_seq;
        float *w_out = p.weights_out + static_cast<size_t>(seg) * p.dst_seq;
        const int m0 = r * R;
        int rows = min(R, n - m0);
        uint4 v[kUnitVecs];
        float w = 0.f;
        int wait_from = 0;   // the units from there on to this one read what this one writes
        if (r < last) {
            const int *kept = p.kept + static_cast<size_t>(seg) * p.k_max;
            for (int i = tid; i < rows; i += kMoveThreads)
                s_at[i] = __ldcg(kept + m0 + i);
            // (positions rise: if the last row is in its place, so are all)
            if (tid == 0)
                s_move = !p.same || __ldcg(kept + m0 + rows - 1) != m0 + rows - 1;
            if (p.in_place && tid == 0) {
                // the first row whose position is m0 or later: of the first rows, positions below are theirs
                int lo = 0, hi = m0;
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    if (__ldcg(kept + mid) >= m0)
                        hi = mid;
                    else
                        lo = mid + 1;
                }
                s_first = lo / R;
            }
            __syncthreads();
            wait_from = p.in_place ? s_first : 0;
            if (!s_move) {   // nothing is stored, nothing has to be waited for
                rows = 0;
                wait_from = r;
            }
#pragma unroll
            for (int k = 0; k < kUnitVecs; ++k) {
                const int i = k * kMoveThreads + tid;          // K's vectors, then V's
                const int kv = i / (R * C), row = i % (R * C) / C, c = i % C;
                if (row < rows)
                    v[k] = __ldcs(reinterpret_cast<const uint4 *>(p.src) +
                                  ((static_cast<size_t>(kv) * segments + seg) * p.src_seq + s_at[row]) * C + c);
            }
            if (tid < rows)
                w = __ldcg(w_in + s_at[tid]);
        }
        if (p.in_place) {
            // (the loads have to have happened, not only been issued, before the flag says so)
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                s_ok = 1;
                if (r < last)
                    st_release(flags + r, 1u);
            }
            __syncthreads();
            for (int u = wait_from + tid; u < min(r, last); u += kMoveThreads) {
                const uint64_t t0 = global_timer_ns();
                while (ld_acquire(flags + u) == 0u) {
                    if (global_timer_ns() - t0 > kWaitLimitNs) {
                        s_ok = 0;
                        atomicOr(p.err, kErrWaitFull);
                        break;
                    }
                }
            }
            __syncthreads();
            if (!s_ok)
                continue;   // nothing is stored over what may not have been read
        }
        if (r < last) {
#pragma unroll
            for (int k = 0; k < kUnitVecs; ++k) {
                const int i = k * kMoveThreads + tid;
                const int kv = i / (R * C), row = i % (R * C) / C, c = i % C;
                if (row < rows)
                    __stcs(reinterpret_cast<uint4 *>(p.dst) +
                               ((static_cast<size_t>(kv) * segments + seg) * p.dst_seq + m0 + row) * C + c,
                           v[k]);
            }
            if (tid < rows)
                w_out[m0 + tid] = w;
        } else {
            for (int u = n + tid; u < p.dst_seq; u += kMoveThreads)
                w_out[u] = 0.f;
        }
    }
}

template <int NT>
const void *keep_fn(int head_dim)
{
    return head_dim == 0    ? reinterpret_cast<const void *>(&keep_kernel<0, NT>)
           : head_dim == 64 ? reinterpret_cast<const void *>(&keep_kernel<64, NT>)
                            : reinterpret_cast<const void *>(&keep_kernel<128, NT>);
}

}  // namespace

int evict_units(int head_dim, int k_max)
{
    const int R = head_dim == 64 ? unit_rows<64>() : unit_rows<128>();
    return (k_max + R - 1) / R + 1;
}

cudaError_t prepare_evict()
{
    cudaError_t e = cudaSuccess;
    for (const void *fn : {keep_fn<kKeepThreads>(0), keep_fn<kKeepThreads>(64), keep_fn<kKeepThreads>(128),
                           keep_fn<kKeepFew>(0), keep_fn<kKeepFew>(64), keep_fn<kKeepFew>(128)})
        if (e == cudaSuccess)
            e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kKeepSmem));
    return e;
}

cudaError_t launch_evict(int head_dim, const EvictParams &p, int max_len, int sm_count, cudaStream_t stream)
{
    int size = 1;
    while (size < kMaxCluster && size * kKeepThreads * 4 < max_len && 2 * p.b * p.g * size <= sm_count)
        size *= 2;
    while (size < kMaxCluster && static_cast<size_t>((max_len + size - 1) / size) * 4 > kKeepSmem)
        size *= 2;
    const size_t keys = static_cast<size_t>((max_len + size - 1) / size) * 4;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.b * p.g * size));
    // Small CTAs where there are more segments than SMs, which then hold four of them (480 of 1000 positions, 250 kept,
    // of 64 channels 15.8 us, 26.1 with large ones; 144 of them 9.4, 6.7 with large ones).
    const bool few = static_cast<long long>(p.b) * p.g > sm_count && max_len <= 8192;
    const int nt = few ? kKeepFew : kKeepThreads;
    cfg.blockDim = dim3(static_cast<unsigned>(nt));
    cfg.dynamicSmemBytes = keys <= kKeepSmem ? keys : kKeepSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(size);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = size > 1 ? 2 : 1;   // (a cluster's launch costs the host a microsecond more)
    void *args[] = {const_cast<EvictParams *>(&p)};
    // One launch where few rounds move what stays of a segment.  A round is a trip to memory and back, the second launch
    // takes 2 to 4 us here and two of the host's.  us into another cache, one / two launches (and in place): 144 segments
    // of 1000 positions, 250 kept, 7.7 / 9.7 (8.2 / 13.7), 16 of 2000, 500 kept (two rounds) 8.6 / 8.3 (10.2 / 12.2), 16
    // of 2000, 1900 kept (eight) 16.8 / 8.8 (23.4 / 15.0); where nearly every SM has a segment, 128 of 2000, 500 kept
    // (four) 17.4 / 18.2 (20.3 / 24.3), of 4000, 1000 kept (eight) 29.2 / 29.4 (36.6 / 39.8).
    const int per_round = size * (nt * kKeepVecs / (head_dim / 4)), rounds = (p.rows + per_round - 1) / per_round;
    const long long ctas = static_cast<long long>(p.b) * p.g * size;
    const bool whole = rounds <= (few || (2 * ctas > sm_count && ctas <= sm_count) ? 4 : ctas <= sm_count ? 2 : 0);
    cudaError_t e = cudaLaunchKernelExC(
        &cfg, few ? keep_fn<kKeepFew>(whole ? head_dim : 0) : keep_fn<kKeepThreads>(whole ? head_dim : 0), args);
    if (e != cudaSuccess || whole)
        return e;
    const long long units = static_cast<long long>(p.b) * p.g * p.units;
    cfg.gridDim = dim3(static_cast<unsigned>(units < 6LL * sm_count ? units : 6LL * sm_count));
    cfg.blockDim = dim3(kMoveThreads);
    cfg.dynamicSmemBytes = 0;
    cfg.numAttrs = 1;
    return cudaLaunchKernelExC(&cfg, head_dim == 64 ? reinterpret_cast<const void *>(&move_kernel<64>)
                                                    : reinterpret_cast<const void *>(&move_kernel<128>), args);
}

}  // namespace mlkv
