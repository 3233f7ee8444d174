// Storing into and reading back the 4-bit KV cache (layout and values: mlkv_q4.h).
//
//   s = bf16(max |x| / 7) over 32 channels, q = the whole number nearest to x / s, halves away from
//   zero.
//
// x and s have 8-bit significands, so x / s is a half exactly or at least 2^-10 away from one (their
// quotient's distance from n + 1/2 is a multiple of 1 / (2 S), S the scale's significand, shifted by
// at most the quotient's own exponent).  x times the approximate reciprocal of s, raised by 2^-16 of
// itself, is therefore on the right side of every half; the sum of its magnitude and 1.5 2^23 rounds it
// and leaves the code's magnitude in the low bits: one multiply-add a channel.  Likewise max |x| times
// fp32(1/7) rounds to the same bf16 as the exact quotient, which is at least 2^-12 of itself away from a
// bf16 midpoint unless it is a bf16.
//
// HBM-bound: 2 bytes a channel on one side, 0.5625 on the other.  Measured on GB300, K and V of 8 sequences
// of 4096 positions, 8 KV heads of 128 (floor 25.3 us each way): store 32.4 us, 5.3 TB/s; read 28.8 us, 6.0
// TB/s.  A batch's new tokens are bound by the call (4.0 us in Python).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "mlkv_q4.h"

#include "mlkv_device.cuh"

namespace mlkv {
namespace {

__device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b)
{
    const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162 *>(&a);
    const __nv_bfloat162 y = *reinterpret_cast<const __nv_bfloat162 *>(&b);
    const __nv_bfloat162 m = __hmax2_nan(__habs2(x), __habs2(y));
    return *reinterpret_cast<const uint32_t *>(&m);
}

// Eight channels of a group whose four lanes are neighbours (lane % 4): their codes as four pairs
// (channels 2 i and 2 i + 1, as q4_pair has them) and the scale's bits.
struct Coded {
    uint32_t p[4];
    uint32_t scale;
};

__device__ __forceinline__ Coded quantise8(uint4 x)
{
    uint32_t m = max_abs2(max_abs2(x.x, x.y), max_abs2(x.z, x.w));
    m = max_abs2(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max_abs2(m, __shfl_xor_sync(0xffffffffu, m, 2));
    m = max_abs2(m, m >> 16);
    const float amax = bf16_lo(m);
    Coded c;
    const float s = __uint_as_float(pack_bf16x2(0.f, amax * (1.f / 7.f)) & 0xffff0000u);
    c.scale = __float_as_uint(s) >> 16;
    float r = fast_rcp(s) * (1.f + 1.f / 65536.f);
    const bool none = !(amax < __int_as_float(0x7f800000)) || s < 1.17549435e-38f;
    if (none)
        c.scale = s < 1.17549435e-38f ? 0u : 0x7fffu;
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // 0x4b40000m: the magnitude is the lowest byte, the next one is 0
        const uint32_t lo = __float_as_uint(fmaf(fabsf(bf16_lo(w[i])), r, 12582912.f));
        const uint32_t hi = __float_as_uint(fmaf(fabsf(bf16_hi(w[i])), r, 12582912.f));
        const uint32_t mags = __byte_perm(lo, hi, 0x4101);
        // without a scale: zeros
        c.p[i] = none ? 0u : (w[i] & 0x80008000u) | mags;
    }
    return c;
}

// A V word from the pairs of 4 channels at the even position (e) and at the odd one (o).
__device__ __forceinline__ uint32_t v_word_of(uint32_t e0, uint32_t e1, uint32_t o0, uint32_t o1)
{
    return q4_word(__byte_perm(e0, o0, 0x5410), __byte_perm(e0, o0, 0x7632),
                   __byte_perm(e1, o1, 0x5410), __byte_perm(e1, o1, 0x7632));
}

// The new token of every (sequence, KV head): a thread per 8 channels.
template <int D>
__global__ void __launch_bounds__(128) q4_append_kernel(const __grid_constant__ Q4StoreParams p)
{
    grid_dependency_wait();
    grid_dependents_launch();
    constexpr int kOct = D / 8;
    const int total = 2 * p.b * p.g * kOct;
    const int idx = blockIdx.x * blockDim.x + threadIdx.x;
    // whole groups of lanes are in or out: total is a multiple of 8
    const bool in = idx < total;
    const int oct = idx % kOct;
    int row = in ? idx / kOct : 0;
    const int bg = p.b * p.g;
    const bool is_v = row >= bg;
    row -= is_v ? bg : 0;
    const uint4 x = *reinterpret_cast<const uint4 *>((is_v ? p.V : p.K) +
                                                     static_cast<size_t>(row) * D + oct * 8);
    uint8_t *dst = p.slot + row * p.row_bytes;
    const int pos = p.seq_len[row / p.g] - 1;
    const Coded c = quantise8(x);
    if (!in)
        return;
    using LY = Q4Layout<D>;
    uint8_t *blk = dst + static_cast<size_t>(pos / kQ4Block) * LY::kBytes;
    const int r = pos % kQ4Block, grp = oct >> 2, t = oct & 3;
    if (is_v) {
        // the words are shared with the pair's other position, whose bits stay
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            uint32_t *at = reinterpret_cast<uint32_t *>(blk + LY::v_word(r, grp, 2 * t + q));
            const uint32_t a = c.p[2 * q], b = c.p[2 * q + 1];
            *at = (*at & ~q4_bits(r & 1)) | ((r & 1) ? v_word_of(0, 0, a, b) : v_word_of(a, b, 0, 0));
        }
    } else {
        *reinterpret_cast<uint32_t *>(blk + LY::k_word(r, grp, t)) =
            q4_word(c.p[0], c.p[1], c.p[2], c.p[3]);
    }
    if (t == 0)
        *reinterpret_cast<uint16_t *>(blk + (is_v ? LY::v_scale(r, grp) : LY::k_scale(r, grp))) =
            static_cast<uint16_t>(c.scale);
}

// Positions of one CTA.  The read: 16 KB each of K and of V (at D = 64 16 x 4096 positions of 4 heads in
// 17.3 us, 18.3 with 64).  The store: 64 (18.3 us there, 19.0 with 128).
constexpr int kStoreTile = 64;
__host__ __device__ constexpr int read_tile(int d) { return 8192 / d; }

// A CTA turns a tile of positions of one (sequence, KV head) into the image of their blocks in shared
// memory and writes it out in 16-byte pieces (the last, partly filled tile: each position to its own
// places, so that positions past it keep their contents).  HBM-bound: 2 bytes a channel in, 0.5625 out.
template <int D>
__global__ void __launch_bounds__(256) q4_store_kernel(const __grid_constant__ Q4StoreParams p)
{
    using LY = Q4Layout<D>;
    constexpr int kOct = D / 8;
    constexpr int kTile = kStoreTile, kImage = kTile / kQ4Block * LY::kBytes;
    constexpr int kTasks = kTile * kOct / 256;   // octets of K (and of V) a thread
    __shared__ __align__(16) uint8_t img[kImage];
    grid_dependency_wait();
    grid_dependents_launch();
    const int tiles = (p.len + kTile - 1) / kTile;
    const int row = static_cast<int>(blockIdx.x) / tiles;
    const int tile = static_cast<int>(blockIdx.x) - row * tiles;
    const int n = min(kTile, p.len - tile * kTile);
    const size_t src = (static_cast<size_t>(row) * p.len + static_cast<size_t>(tile) * kTile) * D;
    uint8_t *dst = p.slot + row * p.row_bytes + static_cast<size_t>(tile) * kImage;
    const int tid = threadIdx.x;
    uint4 x[2][kTasks];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv)
#pragma unroll
        for (int u = 0; u < kTasks; ++u) {
            const int i = u * 256 + tid;
            x[kv][u] = i / kOct < n ? __ldcs(reinterpret_cast<const uint4 *>((kv ? p.V : p.K) + src) + i)
                                    : make_uint4(0, 0, 0, 0);
        }
    constexpr int kStep = 256 / kOct;   // a thread's positions: a step apart, in its own pair's place
    const int oct = tid % kOct, grp = oct >> 2, t = oct & 3;
#pragma unroll
    for (int u = 0; u < kTasks; ++u) {
        const int pos = u * kStep + tid / kOct;
        uint8_t *blk = (n < kTile ? dst : img) + pos / kQ4Block * LY::kBytes;
        const int r = pos % kQ4Block;
        const bool in = pos < n;
        const Coded k = quantise8(x[0][u]), v = quantise8(x[1][u]);
        // The positions of a pair swap quads: the even one stores word 2 t, the odd one 2 t + 1.
        const bool odd = r & 1;
        const uint32_t y0 = __shfl_xor_sync(0xffffffffu, odd ? v.p[0] : v.p[2], kOct);
        const uint32_t y1 = __shfl_xor_sync(0xffffffffu, odd ? v.p[1] : v.p[3], kOct);
        const uint32_t word =
            odd ? v_word_of(y0, y1, v.p[2], v.p[3]) : v_word_of(v.p[0], v.p[1], y0, y1);
        uint32_t *at = reinterpret_cast<uint32_t *>(blk + LY::v_word(r, grp, 2 * t + (odd ? 1 : 0)));
        if (n < kTile) {
            // the prefix ends inside the tile: what lies behind it keeps its bits
            const bool even_in = (pos & ~1) < n, odd_in = (pos | 1) < n;
            const uint32_t keep = (even_in ? 0u : q4_bits(0)) | (odd_in ? 0u : q4_bits(1));
            if (even_in)
                *at = (word & ~keep) | (keep != 0u ? *at & keep : 0u);
        } else {
            *at = word;
        }
        if (in) {
            *reinterpret_cast<uint32_t *>(blk + LY::k_word(r, grp, t)) =
                q4_word(k.p[0], k.p[1], k.p[2], k.p[3]);
            if (t == 0) {
                *reinterpret_cast<uint16_t *>(blk + LY::k_scale(r, grp)) =
                    static_cast<uint16_t>(k.scale);
                *reinterpret_cast<uint16_t *>(blk + LY::v_scale(r, grp)) =
                    static_cast<uint16_t>(v.scale);
            }
        }
    }
    if (n < kTile)
        return;
    __syncthreads();
    for (int i = tid; i < kImage / 16; i += 256)
        reinterpret_cast<uint4 *>(dst)[i] = reinterpret_cast<const uint4 *>(img)[i];
}

// Pair j of a word, times a pair of scales, as bf16: 3 x 8 significant bits, rounded once.  The
// magnitudes become 128 + m in bf16 (their bits in the mantissa), less 128.
__device__ __forceinline__ uint32_t values2(uint32_t w, int j, uint32_t scales)
{
    const uint32_t p = q4_pair(w, j);
    const uint32_t t = (p >> 8 & 0x00070007u) | 0x43004300u;
    const __nv_bfloat162 m = __hadd2(*reinterpret_cast<const __nv_bfloat162 *>(&t),
                                     __floats2bfloat162_rn(-128.f, -128.f));
    const uint32_t v = *reinterpret_cast<const uint32_t *>(&m) | (p & 0x80008000u);
    const __nv_bfloat162 y = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&v),
                                     *reinterpret_cast<const __nv_bfloat162 *>(&scales));
    return *reinterpret_cast<const uint32_t *>(&y);
}

// A CTA brings the blocks of a tile of positions of one (sequence, KV head) into shared memory and writes the
// values of those of [start, start + len), a thread 8 channels of a pair of positions at a time.
template <int D>
__global__ void __launch_bounds__(256) q4_read_kernel(const __grid_constant__ Q4ReadParams p)
{
    using LY = Q4Layout<D>;
    constexpr int kOct = D / 8;
    constexpr int kTile = read_tile(D);
    __shared__ __align__(16) uint8_t img[kTile / kQ4Block * LY::kBytes];
    grid_dependency_wait();
    grid_dependents_launch();
    const int tile0 = p.start / kTile;
    const int tiles = (p.start + p.len - 1) / kTile - tile0 + 1;
    const int row = static_cast<int>(blockIdx.x) / tiles;
    const int pos0 = (tile0 + static_cast<int>(blockIdx.x) - row * tiles) * kTile;
    // the tile's positions [lo, hi) that are asked for, and their blocks
    const int lo = max(p.start - pos0, 0), hi = min(p.start + p.len - pos0, kTile);
    const uint8_t *src =
        p.slot + row * p.row_bytes + static_cast<size_t>(pos0 / kQ4Block) * LY::kBytes;
    const int tid = threadIdx.x;
    const int i1 = ((hi + kQ4Block - 1) / kQ4Block) * LY::kBytes / 16;
    for (int i = lo / kQ4Block * LY::kBytes / 16 + tid; i < i1; i += 256)
        reinterpret_cast<uint4 *>(img)[i] = reinterpret_cast<const uint4 *>(src)[i];
    __syncthreads();
    // pairs [lo / 2, (hi + 1) / 2)
    const int first = lo / 2 * kOct;
    const int n = ((hi + 1) / 2 - lo / 2) * kOct;
    for (int k = tid; k < 2 * n; k += 256) {
        const bool is_v = k >= n;
        const int i = first + (is_v ? k - n : k);
        const int pos = i / kOct * 2, oct = i % kOct, grp = oct >> 2, t = oct & 3;
        const uint8_t *blk = img + pos / kQ4Block * LY::kBytes;
        const int r = pos % kQ4Block;
        uint32_t v[2][4];   // [position][channel pair]
        if (is_v) {
            const uint32_t s = *reinterpret_cast<const uint32_t *>(blk + LY::v_scale(r, grp));
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint32_t w =
                    *reinterpret_cast<const uint32_t *>(blk + LY::v_word(r, grp, 2 * t + q));
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const uint32_t a = values2(w, 2 * c, s);
                    const uint32_t b = values2(w, 2 * c + 1, s);
                    v[0][2 * q + c] = __byte_perm(a, b, 0x5410);
                    v[1][2 * q + c] = __byte_perm(a, b, 0x7632);
                }
            }
        } else {
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                const uint32_t s =
                    *reinterpret_cast<const uint16_t *>(blk + LY::k_scale(r + o, grp)) * 0x10001u;
                const uint32_t w =
                    *reinterpret_cast<const uint32_t *>(blk + LY::k_word(r + o, grp, t));
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    v[o][c] = values2(w, c, s);
            }
        }
        __nv_bfloat16 *dst = (is_v ? p.V : p.K) +
                             (static_cast<long long>(row) * p.len + (pos0 + pos - p.start)) * D +
                             oct * 8;
        if (pos >= lo)
            *reinterpret_cast<uint4 *>(dst) = make_uint4(v[0][0], v[0][1], v[0][2], v[0][3]);
        if (pos + 1 < hi)
            *reinterpret_cast<uint4 *>(dst + D) = make_uint4(v[1][0], v[1][1], v[1][2], v[1][3]);
    }
}

template <typename P>
cudaError_t launch(const void *fn, long long blocks, int threads, const P &p, cudaStream_t stream)
{
    if (blocks > 0x7FFFFFFFLL)
        return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(static_cast<unsigned>(threads));
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    void *args[] = {const_cast<P *>(&p)};
    return cudaLaunchKernelExC(&cfg, fn, args);
}

template <typename F64, typename F128>
const void *pick(int d, F64 *f64, F128 *f128)
{
    return d == 64 ? reinterpret_cast<const void *>(f64) : reinterpret_cast<const void *>(f128);
}

}  // namespace

cudaError_t launch_q4_append(int d, const Q4StoreParams &p, cudaStream_t stream)
{
    const long long total = 2LL * p.b * p.g * (d / 8);
    return launch(pick(d, &q4_append_kernel<64>, &q4_append_kernel<128>), (total + 127) / 128, 128, p,
                  stream);
}

cudaError_t launch_q4_store(int d, const Q4StoreParams &p, cudaStream_t stream)
{
    const long long tiles = (p.len + kStoreTile - 1) / kStoreTile;
    return launch(pick(d, &q4_store_kernel<64>, &q4_store_kernel<128>), tiles * p.b * p.g, 256, p,
                  stream);
}

cudaError_t launch_q4_read(int d, const Q4ReadParams &p, cudaStream_t stream)
{
    const int n = read_tile(d);
    const long long tiles = (p.start + p.len - 1) / n - p.start / n + 1;
    return launch(pick(d, &q4_read_kernel<64>, &q4_read_kernel<128>), tiles * p.b * p.g, 256, p, stream);
}

}  // namespace mlkv
