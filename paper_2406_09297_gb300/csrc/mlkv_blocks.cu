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

// A CTA is one block of one KV head: 16 bytes a load, D / 8 lanes a row, every row of the block in flight at
// once.  Bound by the keys' bytes.
template <int D>
__global__ void __launch_bounds__(kBoundsThreads) bounds_kernel(const __grid_constant__ BoundsParams p)
{
    constexpr int C = D / 8;                     // 16-byte columns of a row
    constexpr int RG = kBoundsThreads / C;       // rows at a time
    constexpr int N = kBlock / RG;               // rows of a thread
    __shared__ float s_lo[RG][D + 4], s_hi[RG][D + 4];
    __shared__ float s_max[kBoundsThreads / 32];
    __shared__ int s_bad;
    const int tid = static_cast<int>(threadIdx.x);
    const int seg = static_cast<int>(blockIdx.x / p.ctas), beta = seg / p.g;
    const int L = p.seq_len[beta];
    const int blk = p.first[beta] / kBlock + static_cast<int>(blockIdx.x % p.ctas);
    if (tid == 0)
        s_bad = 0;
    grid_dependency_wait();
    grid_dependents_launch();
    if (blk * kBlock >= L)
        return;
    const int n = min(kBlock, L - blk * kBlock);
    const int col = tid % C, r0 = tid / C;
    const uint4 *k = reinterpret_cast<const uint4 *>(
                         p.K + (static_cast<size_t>(seg) * p.max_seq + static_cast<size_t>(blk) * kBlock) * D) + col;
    uint4 v[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
        v[i] = k[static_cast<size_t>(min(r0 + i * RG, n - 1)) * C];   // (a row twice changes nothing)
    float lo[8], hi[8];
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        lo[e] = __int_as_float(0x7f800000);
        hi[e] = -lo[e];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = bf16_lo(w[e]), b = bf16_hi(w[e]);
            bad = bad || !(fabsf(a) <= kLargest) || !(fabsf(b) <= kLargest);
            lo[2 * e] = fminf(lo[2 * e], a);
            hi[2 * e] = fmaxf(hi[2 * e], a);
            lo[2 * e + 1] = fminf(lo[2 * e + 1], b);
            hi[2 * e + 1] = fmaxf(hi[2 * e + 1], b);
        }
    }
    __syncthreads();
    if (bad)
        s_bad = 1;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        s_lo[r0][col * 8 + e] = lo[e];
        s_hi[r0][col * 8 + e] = hi[e];
    }
    __syncthreads();
    float a = 0.f, b = 0.f, amax = 0.f;
    if (tid < D) {
        a = s_lo[0][tid];
        b = s_hi[0][tid];
        for (int r = 1; r < RG; ++r) {
            a = fminf(a, s_lo[r][tid]);
            b = fmaxf(b, s_hi[r][tid]);
        }
        amax = fmaxf(fabsf(a), fabsf(b));
    }
    for (int s = 16; s > 0; s >>= 1)
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, s));
    if ((tid & 31) == 0)
        s_max[tid >> 5] = amax;
    __syncthreads();
    amax = 0.f;
    for (int w = 0; w < kBoundsThreads / 32; ++w)
        amax = fmaxf(amax, s_max[w]);
    const bool unknown = s_bad != 0;
    const float scale = unknown ? __int_as_float(0x7f800000) : scale_of(amax);
    const size_t at = static_cast<size_t>(seg) * p.n_blocks + blk;
    if (tid < D) {
        const float inv = unknown ? 0.f : inverse_power(scale);   // exact quotients
        p.bounds[at * 2 * D + tid] = unknown ? -127 : static_cast<int8_t>(floorf(a * inv));
        p.bounds[at * 2 * D + D + tid] = unknown ? 127 : static_cast<int8_t>(ceilf(b * inv));
    }
    if (tid == 0)
        p.scales[at] = scale;
}

// A cluster is one (sequence, KV head): each CTA scores a run of its blocks, a thread a block (dp4a of the
// codes with the query's positive and negative parts), keeps the scores as ordered keys in shared memory, and
// the cluster takes the largest (cluster_topk).  Bound by latency for few blocks, else by the bounds' bytes.
template <int D>
__global__ void __launch_bounds__(kTopkThreads) select_kernel(const __grid_constant__ SelectParams p)
{
    namespace cg = cooperative_groups;
    __shared__ TopkShared sh;
    __shared__ __align__(16) uint32_t s_q[2][MLKV_MAX_GROUP][D / 4];   // positive, negative part
    __shared__ float s_f[MLKV_MAX_GROUP];                              // 2^f, 0: no say
    extern __shared__ unsigned s_key[];
    cg::cluster_group cluster = cg::this_cluster();
    const int size = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int seg = static_cast<int>(blockIdx.x) / size;
    const int beta = seg / p.g, j = seg - beta * p.g;
    const int tid = static_cast<int>(threadIdx.x), lane = tid & 31, warp = tid >> 5;
    const int count = (p.seq_len[beta] + kBlock - 1) / kBlock;
    const int per = (count + size - 1) / size;
    const int first = min(count, rank * per), n = min(count, first + per) - first;
    int *to = p.blocks + static_cast<size_t>(seg) * p.n_select;
    grid_dependency_wait();
    grid_dependents_launch();
    if (count <= p.n_select) {   // all of them
        for (int i = rank * kTopkThreads + tid; i < p.n_select; i += size * kTopkThreads)
            to[i] = i < count ? i : -1;
        return;
    }
    const __nv_bfloat16 *q = p.Q + (static_cast<size_t>(beta) * p.h + static_cast<size_t>(j) * p.G) * D;
    for (int i = warp; i < p.G; i += kTopkThreads / 32) {
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
    for (int i = tid; i < n; i += kTopkThreads) {
        const int blk = first + i;
        unsigned key = 0xffffffffu;   // selected in any case
        if (blk >= p.n_first && blk < count - p.n_last) {
            const size_t at = static_cast<size_t>(seg) * p.n_blocks + blk;
            const uint4 *lo = reinterpret_cast<const uint4 *>(p.bounds + at * 2 * D), *hi = lo + D / 16;
            const float scale = p.scales[at];
            float best = -__int_as_float(0x7f800000);
            int sum[MLKV_MAX_GROUP];
#pragma unroll
            for (int a = 0; a < MLKV_MAX_GROUP; ++a)
                sum[a] = 0;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                const uint4 l4 = lo[c], h4 = hi[c];
#pragma unroll
                for (int a = 0; a < MLKV_MAX_GROUP; ++a) {
                    if (a >= p.G)
                        break;
                    const uint4 qp = *reinterpret_cast<const uint4 *>(&s_q[0][a][c * 4]);
                    const uint4 qn = *reinterpret_cast<const uint4 *>(&s_q[1][a][c * 4]);
                    int t = sum[a];
                    t = __dp4a(static_cast<int>(qp.x), static_cast<int>(h4.x), t);
                    t = __dp4a(static_cast<int>(qp.y), static_cast<int>(h4.y), t);
                    t = __dp4a(static_cast<int>(qp.z), static_cast<int>(h4.z), t);
                    t = __dp4a(static_cast<int>(qp.w), static_cast<int>(h4.w), t);
                    t = __dp4a(static_cast<int>(qn.x), static_cast<int>(l4.x), t);
                    t = __dp4a(static_cast<int>(qn.y), static_cast<int>(l4.y), t);
                    t = __dp4a(static_cast<int>(qn.z), static_cast<int>(l4.z), t);
                    t = __dp4a(static_cast<int>(qn.w), static_cast<int>(l4.w), t);
                    sum[a] = t;
                }
            }
            const bool unknown = scale == __int_as_float(0x7f800000);
#pragma unroll
            for (int a = 0; a < MLKV_MAX_GROUP; ++a)
                if (a < p.G && s_f[a] != 0.f)
                    best = fmaxf(best, static_cast<float>(sum[a]) * (s_f[a] * scale));
            // ordered: negative numbers below positive ones, both zeros alike
            const uint32_t u = __float_as_uint(best + 0.f);
            key = unknown ? 0xfffffffeu : (u >> 31) ? ~u : u | 0x80000000u;
        }
        s_key[i] = key;
    }
    __syncthreads();
    cluster_topk(sh, n, static_cast<unsigned>(p.n_select), [&](int i) { return s_key[i]; },
                 [&](unsigned place, int i) { to[place] = first + i; });
}

constexpr int kMaxCluster = 8;
constexpr size_t kSelectSmem = 160 * 1024;

template <int D>
const void *select_fn()
{
    return reinterpret_cast<const void *>(&select_kernel<D>);
}

}  // namespace

cudaError_t launch_bounds(int head_dim, const BoundsParams &p, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.ctas * static_cast<unsigned>(p.b * p.g));
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

int select_max_blocks() { return kMaxCluster * static_cast<int>(kSelectSmem / 4); }

cudaError_t prepare_select(int head_dim)
{
    return cudaFuncSetAttribute(head_dim == 64 ? select_fn<64>() : select_fn<128>(),
                                cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSelectSmem));
}

cudaError_t launch_select(int head_dim, const SelectParams &p, int max_blocks, cudaStream_t stream)
{
    // CTAs of a cluster: a block a thread where there are that few, fewer CTAs where the clusters alone fill
    // the GPU.
    int size = 1;
    while (size < kMaxCluster && size * kTopkThreads < max_blocks && p.b * p.g * size < 304)
        size *= 2;
    while (size < kMaxCluster && static_cast<size_t>((max_blocks + size - 1) / size) * 4 > kSelectSmem)
        size *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.b * p.g * size));
    cfg.blockDim = dim3(kTopkThreads);
    cfg.dynamicSmemBytes = static_cast<size_t>((max_blocks + size - 1) / size) * 4;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(size);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    void *args[] = {const_cast<SelectParams *>(&p)};
    return cudaLaunchKernelExC(&cfg, head_dim == 64 ? select_fn<64>() : select_fn<128>(), args);
}

}  // namespace mlkv
