// Bounds of the keys of blocks of 64 positions, and the blocks that they promise the largest scores, for GB300.
//
// A block's bounds: with amax the largest |k| of its visible positions and channels, scale = 2^e, e the least
// whole number in [-60, 40] with amax <= 127 * 2^e, and for every channel the codes floor(min / scale) and
// ceil(max / scale), in [-127, 127].  A block with a NaN, an infinity or more than 127 * 2^40 has scale infinity
// and codes -127 and 127: nothing is known of it, and it is taken first.
// A query head in 8 bits: q8 = q / 2^f to the nearest, halves to even, f as e but of the head; a head with
// a NaN, an infinity or more than 127 * 2^40 has no say.  A block's score for the head is
//   2^f scale sum_c max(q8_c lo_c, q8_c hi_c),
// no less (but for the query's rounding) than the score of any key in the block.  The sum is a whole number below
// 128 * 127^2 < 2^21 and the factor a power of two within [2^-120, 2^80]: exact in 32 bits, in any order, so that
// a selection does not depend on how it was computed.
#include "mlkv_device.cuh"
#include "mlkv_long.h"
#include "mlkv_topk.cuh"

namespace mlkv {
namespace {

constexpr float kLargest = 127.f * 1099511627776.f;   // 127 * 2^40

// 2^e for the least e in [-60, 40] with amax <= 127 * 2^e, of a finite bf16 amax <= 127 * 2^40: with
// amax = 1.f * 2^E that is E - 6, but E - 5 where 1.f exceeds 127 / 64 (f = 127 of 128).
__device__ __forceinline__ float scale_of(float amax)
{
    const uint32_t u = __float_as_uint(amax);
    const int E = static_cast<int>(u >> 23) - 127;
    int e = E - 6 + (((u >> 16) & 127u) == 127u ? 1 : 0);
    e = max(e, -60);
    return __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}
// (E of zero and of subnormal numbers is -127: below -60 as well.)

__device__ __forceinline__ float inverse_power(float s)   // of a power of two
{
    return __uint_as_float((254u << 23) - __float_as_uint(s));
}

constexpr int kBoundsThreads = 128;
constexpr int kBoundsCtas = 5;     // an SM

// A warp has a block at a time, half a block of 128 channels on the way at once: 16 bytes a load, D / 8 lanes a row.
// Minima and maxima two channels at a time, NaNs kept, so that the largest magnitude is found among them at the end;
// across rows by shuffles, without shared memory or barriers.  Bound by the keys' bytes: 8 uneven
// sequences of up to 16,000 positions, 8 KV heads of 128, 218 MB, 34.3 us, 6.35 TB/s; 16 of 131,072, one KV head of 64,
// 268 MB, 40.7 us.  (Four warps a block, two blocks after one another, sums through shared memory: 34.9 and 48.7 us.)
template <int D>
__global__ void __launch_bounds__(kBoundsThreads, kBoundsCtas) bounds_kernel(const __grid_constant__ BoundsParams p)
{
    constexpr int C = D / 8;                     // 16-byte columns of a row
    constexpr int R = 32 / C;                    // rows of a warp's load
    constexpr int N = 16;                        // loads on the way
    constexpr int W = kBoundsThreads / 32;
    const int warp = static_cast<int>(threadIdx.x) >> 5, lane = static_cast<int>(threadIdx.x) & 31;
    // the sequence whose CTAs these are
    int beta = 0, above = p.b - 1;
    while (beta < above) {
        const int mid = (beta + above + 1) >> 1;
        if (p.start[mid] <= static_cast<int>(blockIdx.x))
            beta = mid;
        else
            above = mid - 1;
    }
    const int L = p.seq_len[beta], blk0 = p.first[beta] / kBlock, n_blk = (L + kBlock - 1) / kBlock;
    const int ctas = (n_blk - blk0 + p.per_cta - 1) / p.per_cta;   // of a KV head
    const int rel = static_cast<int>(blockIdx.x) - p.start[beta];
    const int j = rel / ctas, at0 = blk0 + (rel - j * ctas) * p.per_cta;
    const size_t seg = static_cast<size_t>(beta) * p.g + j;
    const int col = lane % C, r0 = lane / C;
    grid_dependency_wait();
    grid_dependents_launch();
    for (int blk = at0 + warp; blk < min(n_blk, at0 + p.per_cta); blk += W) {
        const int n = min(kBlock, L - blk * kBlock);   // visible positions
        const uint4 *k = reinterpret_cast<const uint4 *>(
                             p.K + (seg * p.max_seq + static_cast<size_t>(blk) * kBlock) * D) + col;
        __nv_bfloat162 lo[4], hi[4];
#pragma unroll
        for (int half = 0; half < kBlock / (N * R); ++half) {
            uint4 v[N];
#pragma unroll
            for (int i = 0; i < N; ++i)   // (a row twice changes nothing)
                v[i] = k[static_cast<size_t>(min(r0 + (half * N + i) * R, n - 1)) * C];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const __nv_bfloat162 *x = reinterpret_cast<const __nv_bfloat162 *>(&v[i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    lo[e] = half + i == 0 ? x[e] : __hmin2_nan(lo[e], x[e]);
                    hi[e] = half + i == 0 ? x[e] : __hmax2_nan(hi[e], x[e]);
                }
            }
        }
        auto other = [](__nv_bfloat162 x, int s) {
            const uint32_t u = __shfl_xor_sync(0xffffffffu, *reinterpret_cast<const uint32_t *>(&x), s);
            return *reinterpret_cast<const __nv_bfloat162 *>(&u);
        };
#pragma unroll
        for (int s = C; s < 32; s <<= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                lo[e] = __hmin2_nan(lo[e], other(lo[e], s));
                hi[e] = __hmax2_nan(hi[e], other(hi[e], s));
            }
        __nv_bfloat162 amax = __habs2(lo[0]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            amax = __hmax2_nan(amax, __hmax2_nan(__habs2(lo[e]), __habs2(hi[e])));
        // (as whole numbers, the bits of magnitudes are in their order, NaN last)
        const uint32_t bits = *reinterpret_cast<const uint32_t *>(&amax);
        const float most = __uint_as_float(__reduce_max_sync(0xffffffffu, max(bits << 16, bits & 0xffff0000u)));
        const bool unknown = !(most <= kLargest);
        const float scale = unknown ? __int_as_float(0x7f800000) : scale_of(most);
        const size_t at = seg * p.n_blocks + blk;
        // eight channels a lane: the first row's lanes their least codes, the second row's their largest, as -floor(-y)
        if (r0 < 2) {
            const float inv = (unknown ? 0.f : inverse_power(scale)) * (r0 == 1 ? -1.f : 1.f);   // exact quotients
            uint32_t codes[2] = {0u, 0u};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 y = __bfloat1622float2(r0 == 1 ? hi[e] : lo[e]);
                const int a = unknown ? -127 : __float2int_rd(y.x * inv), b = unknown ? -127 : __float2int_rd(y.y * inv);
                codes[e / 2] |= ((static_cast<uint32_t>(r0 == 1 ? -a : a) & 255u) |
                                 ((static_cast<uint32_t>(r0 == 1 ? -b : b) & 255u) << 8)) << (16 * (e % 2));
            }
            *reinterpret_cast<uint2 *>(p.bounds + at * 2 * D + r0 * D + col * 8) = make_uint2(codes[0], codes[1]);
        }
        if (lane == 0)
            p.scales[at] = scale;
    }
}

constexpr int kSelectThreads = 512;
constexpr int kLanes = 4;   // lanes of a block's score

// A cluster is one (sequence, KV head): each CTA scores a run of its blocks, four lanes a block (dp4a of the
// codes with the query's positive and negative parts; 64 bytes a load), and puts the scores as ordered keys into
// the first CTA's shared memory, which takes the largest (cluster_topk).  Bound by latency for few blocks (2048 blocks of
// one KV head, 12 heads of 64, 11 us), else by the products, 2 D / 4 dp4a a block and head (32 uneven sequences of up to 512
// blocks, 8 KV heads, 4 heads of 128 each, 12.5 us).
template <int D>
__global__ void __launch_bounds__(kSelectThreads) select_kernel(const __grid_constant__ SelectParams p)
{
    namespace cg = cooperative_groups;
    constexpr int NT = kSelectThreads, C = D / 16 / kLanes;   // 16-byte columns of a lane
    __shared__ TopkShared<NT> sh;
    __shared__ unsigned s_mm[2 * NT / 32];
    __shared__ __align__(16) uint32_t s_q[2][MLKV_MAX_GROUP][D / 4];   // positive, negative part
    __shared__ float s_f[MLKV_MAX_GROUP];                              // 2^f, 0: no say
    extern __shared__ unsigned s_key[];
    cg::cluster_group cluster = cg::this_cluster();
    const int size = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int seg = static_cast<int>(blockIdx.x) / size;
    const int beta = seg / p.g, j = seg - beta * p.g;
    const int tid = static_cast<int>(threadIdx.x), lane = tid & 31, warp = tid >> 5;
    const int count = (p.seq_len[beta] + kBlock - 1) / kBlock;
    int *to = p.blocks + static_cast<size_t>(seg) * p.n_select;
    grid_dependency_wait();
    grid_dependents_launch();
    if (count <= p.n_select) {   // all of them
        for (int i = rank * NT + tid; i < p.n_select; i += size * NT)
            to[i] = i < count ? i : -1;
        return;
    }
    // the blocks at either end, which are selected in any case
    if (rank == 0)
        for (int i = tid; i < p.n_first + p.n_last; i += NT)
            to[i < p.n_first ? i : p.n_select - p.n_last + i - p.n_first] =
                i < p.n_first ? i : count - p.n_last + i - p.n_first;
    const int want = p.n_select - p.n_first - p.n_last;
    if (want == 0)
        return;
    if (size > 1)
        cluster_arrive();   // (the first CTA's shared memory is there once all have started)
    const int inner = count - p.n_first - p.n_last, per = (inner + size - 1) / size;
    const int first = p.n_first + min(inner, rank * per), n = min(inner, (rank + 1) * per) - min(inner, rank * per);
    // a lane's columns of its first block, on the way while the queries are made ready
    const int part = tid % kLanes;
    const size_t base = static_cast<size_t>(seg) * p.n_blocks + first;
    uint4 lo4[C], hi4[C];
    float scale = 0.f;
    auto fetch = [&](int i) {
        if (i >= n)
            return;
        const uint4 *lo = reinterpret_cast<const uint4 *>(p.bounds + (base + i) * 2 * D), *hi = lo + D / 16;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            lo4[c] = lo[c * kLanes + part];
            hi4[c] = hi[c * kLanes + part];
        }
        scale = p.scales[base + i];
    };
    fetch(tid / kLanes);
    const __nv_bfloat16 *q = p.Q + (static_cast<size_t>(beta) * p.h + static_cast<size_t>(j) * p.G) * D;
    for (int i = warp; i < p.G; i += NT / 32) {
        constexpr int E = D / 32;
        float x[E], amax = 0.f;
        bool bad = false;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            x[e] = __bfloat162float(q[i * D + lane * E + e]);
            bad = bad || !(fabsf(x[e]) <= kLargest);
            amax = fmaxf(amax, fabsf(x[e]));
        }
        bad = __any_sync(0xffffffffu, bad);
        for (int s = 16; s > 0; s >>= 1)
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, s));
        const float f = bad ? 0.f : scale_of(amax), inv = bad ? 0.f : inverse_power(f);
        int8_t *pos = reinterpret_cast<int8_t *>(s_q[0][i]), *neg = reinterpret_cast<int8_t *>(s_q[1][i]);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = bad ? 0 : __float2int_rn(x[e] * inv);
            pos[lane * E + e] = static_cast<int8_t>(max(c, 0));
            neg[lane * E + e] = static_cast<int8_t>(min(c, 0));
        }
        if (lane == 0)
            s_f[i] = f;
    }
    __syncthreads();
    unsigned *keys = size > 1 ? cluster.map_shared_rank(s_key, 0) + (first - p.n_first) : s_key;
    if (size > 1)
        cluster_wait();
    const int per_round = NT / kLanes;
    for (int i0 = 0; i0 < n; i0 += per_round) {   // (all lanes stay: they add up in groups)
        const int i = i0 + tid / kLanes;
        float best = -__int_as_float(0x7f800000);
        for (int a = 0; a < p.G; ++a) {
            int t = 0;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const uint4 qp = *reinterpret_cast<const uint4 *>(&s_q[0][a][(c * kLanes + part) * 4]);
                const uint4 qn = *reinterpret_cast<const uint4 *>(&s_q[1][a][(c * kLanes + part) * 4]);
                t = __dp4a(static_cast<int>(qp.x), static_cast<int>(hi4[c].x), t);
                t = __dp4a(static_cast<int>(qp.y), static_cast<int>(hi4[c].y), t);
                t = __dp4a(static_cast<int>(qp.z), static_cast<int>(hi4[c].z), t);
                t = __dp4a(static_cast<int>(qp.w), static_cast<int>(hi4[c].w), t);
                t = __dp4a(static_cast<int>(qn.x), static_cast<int>(lo4[c].x), t);
                t = __dp4a(static_cast<int>(qn.y), static_cast<int>(lo4[c].y), t);
                t = __dp4a(static_cast<int>(qn.z), static_cast<int>(lo4[c].z), t);
                t = __dp4a(static_cast<int>(qn.w), static_cast<int>(lo4[c].w), t);
            }
#pragma unroll
            for (int s = 1; s < kLanes; s <<= 1)
                t += __shfl_xor_sync(0xffffffffu, t, s);
            if (s_f[a] != 0.f)
                best = fmaxf(best, static_cast<float>(t) * (s_f[a] * scale));
        }
        if (i < n) {
            // ordered: negative numbers below positive ones, both zeros alike; nothing known: before all
            const uint32_t u = __float_as_uint(best + 0.f);
            const unsigned key = scale == __int_as_float(0x7f800000) ? 0xffffffffu
                                 : (u >> 31)                         ? ~u
                                                                     : u | 0x80000000u;
            if (part == 0)
                keys[i] = key;
        }
        fetch(i + per_round);
    }
    if (size > 1) {
        cluster.sync();
        if (rank != 0)
            return;
    } else {
        __syncthreads();
    }
    unsigned least = 0xffffffffu, most = 0u;
    for (int i = tid; i < inner; i += NT) {
        least = min(least, s_key[i]);
        most = max(most, s_key[i]);
    }
    block_min_max<NT>(least, most, s_mm);
    cluster_topk<NT>(sh, 1, 0, inner, least, most, static_cast<unsigned>(want), [&](int i) { return s_key[i]; },
                     [&](unsigned place, int i) { to[p.n_first + place] = p.n_first + i; });
}

constexpr int kMaxCluster = kTopkCluster;
constexpr size_t kSelectSmem = 128 * 1024;   // keys of a (sequence, KV head)

template <int D>
const void *select_fn()
{
    return reinterpret_cast<const void *>(&select_kernel<D>);
}

}  // namespace

// Blocks of a CTA: one a warp if the GPU holds them all at once, else two, which spares CTAs' starts (480 blocks of 64
// channels 2.9 us, 3.3 with two a warp).
int bounds_per_cta(long long blocks, int sm_count)
{
    constexpr int W = kBoundsThreads / 32;
    return blocks <= static_cast<long long>(W) * kBoundsCtas * sm_count ? W : 2 * W;
}

cudaError_t launch_bounds(int head_dim, const BoundsParams &p, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.start[p.b]));
    cfg.blockDim = dim3(kBoundsThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    void *args[] = {const_cast<BoundsParams *>(&p)};
    return cudaLaunchKernelExC(&cfg, head_dim == 64 ? reinterpret_cast<const void *>(&bounds_kernel<64>)
                                                    : reinterpret_cast<const void *>(&bounds_kernel<128>), args);
}

int select_max_blocks() { return static_cast<int>(kSelectSmem / 4); }

cudaError_t prepare_select(int head_dim)
{
    return cudaFuncSetAttribute(head_dim == 64 ? select_fn<64>() : select_fn<128>(),
                                cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSelectSmem));
}

cudaError_t launch_select(int head_dim, const SelectParams &p, int max_blocks, cudaStream_t stream)
{
    // CTAs of a cluster: two rounds of scores each, fewer CTAs where the clusters alone fill the GPU.
    int size = 1;
    while (size < kMaxCluster && size * 256 < max_blocks && p.b * p.g * size < 152)
        size *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.b * p.g * size));
    cfg.blockDim = dim3(kSelectThreads);
    cfg.dynamicSmemBytes = static_cast<size_t>(max_blocks) * 4;   // (of use to a cluster's first CTA alone)
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(size);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = size > 1 ? 2 : 1;   // (a cluster's launch costs the host a microsecond more)
    void *args[] = {const_cast<SelectParams *>(&p)};
    return cudaLaunchKernelExC(&cfg, head_dim == 64 ? select_fn<64>() : select_fn<128>(), args);
}

}  // namespace mlkv
