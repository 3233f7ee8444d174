// Queries, keys and values of a projection made ready for the cache's calls (mlkv_qk_norm_rope): RMS
// norm of every query and key head, rotary position encoding in the same pass, values moved along.
//
//   y = x / sqrt(mean(x^2) + eps) * gain           per head, over its D channels
//   (a, b) -> (a cos - b sin, b cos + a sin)       on the first rot channels, (a, b) = channels i and
//                                                  i + rot/2, or 2i and 2i + 1 (interleaved)
//
// In fp32, rounded once, to bf16.  Every channel is read once and written once, so HBM bounds it (per
// channel 4 bytes against ~12 operations); a head is D / 8 lanes of 16 bytes each, whose square sums
// and rotation partners are exchanged with shuffles.  A warp takes U x (256 / D) heads of one token: the
// token's row of the table and the gains are loaded once for all of them and U loads are in flight per
// lane.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <cmath>

#include "mlkv_host.h"

#include "mlkv_device.cuh"

namespace mlkv {
namespace {

struct NormRopeParams {
    const __nv_bfloat16 *Q, *K, *V;            // token rows of h, g, g heads, strides apart
    long long q_stride, k_stride, v_stride;    // elements
    const __nv_bfloat16 *q_gain, *k_gain;      // [D] or null
    const float *cos, *sin;                    // [n_pos][rot / 2]
    const int *positions;                      // [tokens]
    __nv_bfloat16 *q_out;                      // [b][s][h][D]
    __nv_bfloat16 *k_out, *v_out;              // [b][g][s][D]
    float eps;
    int tokens, s, h, g, heads;                // heads: h + g, and g more with V
    int rot, n_pos, interleaved, chunks;       // chunks: warps per token
};

constexpr int kNormThreads = 128;

template <int D, int U>
__global__ void __launch_bounds__(kNormThreads)
    norm_rope_kernel(const __grid_constant__ NormRopeParams p)
{
    constexpr int LPH = D / 8;        // lanes per head, 8 channels each
    constexpr int HPI = 32 / LPH;     // heads per warp-wide load
    grid_dependency_wait();
    grid_dependents_launch();
    const int lane = threadIdx.x & 31;
    const long long w = static_cast<long long>(blockIdx.x) * (kNormThreads / 32) + (threadIdx.x >> 5);
    const long long token = w / p.chunks;
    if (token >= p.tokens)
        return;
    const int c = static_cast<int>(w - token * p.chunks);
    const int sub = lane % LPH;       // channels 8 sub .. 8 sub + 7
    const int hd0 = c * U * HPI + lane / LPH;
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int hd = hd0 + u * HPI;
        const __nv_bfloat16 *src = nullptr;
        if (hd < p.h)
            src = p.Q + token * p.q_stride + hd * D;
        else if (hd < p.h + p.g)
            src = p.K + token * p.k_stride + (hd - p.h) * D;
        else if (hd < p.heads)
            src = p.V + token * p.v_stride + (hd - p.h - p.g) * D;
        x[u] = src != nullptr ? *reinterpret_cast<const uint4 *>(src + sub * 8)
                              : make_uint4(0, 0, 0, 0);
    }
    // The token's rotation of this lane's channels: y[i] cos[i] + other[i] sin[i], sin signed.
    const int hc = p.rot / 16;        // 8-channel pieces of half the rotated channels
    const bool rotates = sub < 2 * hc;
    const bool low = sub < hc;
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        cs[i] = 1.f;
        sn[i] = 0.f;
    }
    if (rotates) {
        const int pos = p.positions[token];
        if (pos >= 0 && pos < p.n_pos) {
            if (p.interleaved) {
                // pairs of neighbours: 4 table entries for 8 channels
                const size_t at = static_cast<size_t>(pos) * (p.rot / 2) + sub * 4;
                const float4 a = *reinterpret_cast<const float4 *>(p.cos + at);
                const float4 b = *reinterpret_cast<const float4 *>(p.sin + at);
                const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    cs[i] = av[i / 2];
                    sn[i] = (i & 1) ? bv[i / 2] : -bv[i / 2];
                }
            } else {
                const size_t at =
                    static_cast<size_t>(pos) * (p.rot / 2) + (low ? sub : sub - hc) * 8;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const float4 a = *reinterpret_cast<const float4 *>(p.cos + at + 4 * q);
                    const float4 b = *reinterpret_cast<const float4 *>(p.sin + at + 4 * q);
                    cs[4 * q] = a.x;
                    cs[4 * q + 1] = a.y;
                    cs[4 * q + 2] = a.z;
                    cs[4 * q + 3] = a.w;
                    sn[4 * q] = low ? -b.x : b.x;
                    sn[4 * q + 1] = low ? -b.y : b.y;
                    sn[4 * q + 2] = low ? -b.z : b.z;
                    sn[4 * q + 3] = low ? -b.w : b.w;
                }
            }
        } else {
            // outside the table: the rotated channels say so
#pragma unroll
            for (int i = 0; i < 8; ++i)
                cs[i] = __int_as_float(0x7fffffff);
        }
    }
    uint4 gq = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u), gk = gq;
    if (p.q_gain != nullptr)
        gq = *reinterpret_cast<const uint4 *>(p.q_gain + sub * 8);
    if (p.k_gain != nullptr)
        gk = *reinterpret_cast<const uint4 *>(p.k_gain + sub * 8);
    const int partner = (lane & ~(LPH - 1)) | (rotates ? (low ? sub + hc : sub - hc) : sub);
    const long long beta = token / p.s;
    const long long t = token - beta * p.s;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int hd = hd0 + u * HPI;
        const bool is_q = hd < p.h, is_v = hd >= p.h + p.g;
        float y[8] = {bf16_lo(x[u].x), bf16_hi(x[u].x), bf16_lo(x[u].y), bf16_hi(x[u].y),
                      bf16_lo(x[u].z), bf16_hi(x[u].z), bf16_lo(x[u].w), bf16_hi(x[u].w)};
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            ss = fmaf(y[i], y[i], ss);
#pragma unroll
        for (int m = 1; m < LPH; m <<= 1)
            ss += __shfl_xor_sync(0xffffffffu, ss, m);
        const float inv = rsqrtf(ss * (1.f / D) + p.eps);
        const uint4 gw = is_q ? gq : gk;
        const float gain[8] = {bf16_lo(gw.x), bf16_hi(gw.x), bf16_lo(gw.y), bf16_hi(gw.y),
                               bf16_lo(gw.z), bf16_hi(gw.z), bf16_lo(gw.w), bf16_hi(gw.w)};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            y[i] = y[i] * inv * gain[i];
        float r[8];
        if (p.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                r[i] = fmaf(y[i ^ 1], sn[i], y[i] * cs[i]);
        } else if (hc > 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float o = __shfl_sync(0xffffffffu, y[i], partner);
                r[i] = fmaf(o, sn[i], y[i] * cs[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                r[i] = y[i];
        }
        uint4 v = make_uint4(pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]),
                             pack_bf16x2(r[4], r[5]), pack_bf16x2(r[6], r[7]));
        if (is_v)
            v = x[u];
        if (hd < p.heads) {
            __nv_bfloat16 *dst;
            if (is_q) {
                dst = p.q_out + (token * p.h + hd) * D;
            } else {
                const int j = hd - p.h - (is_v ? p.g : 0);
                dst = (is_v ? p.v_out : p.k_out) + ((beta * p.g + j) * p.s + t) * D;
            }
            *reinterpret_cast<uint4 *>(dst + sub * 8) = v;
        }
    }
}

template <int D, int U>
const void *norm_fn()
{
    return reinterpret_cast<const void *>(&norm_rope_kernel<D, U>);
}

}  // namespace
}  // namespace mlkv

extern "C" int mlkv_qk_norm_rope(const void *Q, const void *K, const void *V, int64_t q_stride,
                                 int64_t k_stride, int64_t v_stride, const void *q_gain,
                                 const void *k_gain, const float *cos_table,
                                 const float *sin_table, int n_pos, int rot_dim, int interleaved,
                                 const int *positions, float eps, int batch, int s, int n_q_heads,
                                 int kv_heads, int head_dim, void *Q_out, void *K_out, void *V_out,
                                 void *cuda_stream)
{
    using namespace mlkv;
    if (Q == nullptr || K == nullptr || Q_out == nullptr || K_out == nullptr)
        return fail(MLKV_ERR_INVALID_ARG, "Q, K, Q_out and K_out must be non-NULL");
    if ((V == nullptr) != (V_out == nullptr))
        return fail(MLKV_ERR_INVALID_ARG, "V and V_out must both be given or both be NULL");
    if (batch < 1 || s < 1 || n_q_heads < 1 || kv_heads < 1)
        return fail(MLKV_ERR_INVALID_ARG, "sizes must be positive (batch=%d s=%d h=%d g=%d)", batch,
                    s, n_q_heads, kv_heads);
    if (head_dim != 64 && head_dim != 128)
        return fail(MLKV_ERR_UNSUPPORTED, "head_dim %d: this build supports 64 and 128", head_dim);
    for (const void *x : {Q, K, V, q_gain, k_gain, static_cast<const void *>(Q_out),
                          static_cast<const void *>(K_out), static_cast<const void *>(V_out),
                          static_cast<const void *>(cos_table), static_cast<const void *>(sin_table)})
        if (!aligned16(x))
            return fail(MLKV_ERR_INVALID_ARG, "every tensor must be 16-byte aligned");
    for (const int64_t st : {q_stride, k_stride, v_stride})
        if (st < 0 || st % 8 != 0)
            return fail(MLKV_ERR_INVALID_ARG, "a token stride must be a multiple of 8 elements");
    if (rot_dim < 0 || rot_dim > head_dim)
        return fail(MLKV_ERR_INVALID_ARG, "rot_dim %d outside [0, %d]", rot_dim, head_dim);
    if (rot_dim % 16 != 0)
        return fail(MLKV_ERR_UNSUPPORTED, "rot_dim %d: this build supports multiples of 16", rot_dim);
    if (rot_dim > 0 && (cos_table == nullptr || sin_table == nullptr || positions == nullptr))
        return fail(MLKV_ERR_INVALID_ARG, "the rotary tables and positions must be non-NULL");
    if (rot_dim > 0 && n_pos < 1)
        return fail(MLKV_ERR_INVALID_ARG, "n_pos %d must be positive", n_pos);
    if ((reinterpret_cast<uintptr_t>(positions) & 3u) != 0)
        return fail(MLKV_ERR_INVALID_ARG, "positions must be 4-byte aligned");
    if (!(eps >= 0.f) || std::isinf(eps))
        return fail(MLKV_ERR_INVALID_ARG, "eps must be finite and not negative");
    const long long tokens = static_cast<long long>(batch) * s;
    const long long heads = static_cast<long long>(n_q_heads) + (V != nullptr ? 2LL : 1LL) * kv_heads;
    if (tokens > 0x7fffffffLL || heads > (1 << 20))
        return fail(MLKV_ERR_UNSUPPORTED, "%lld tokens of %lld heads exceed what one call takes",
                    tokens, heads);
    // Outputs may not share memory with inputs or each other, but for one that is its own input, row
    // for row (each warp then reads a head before it writes it).
    const size_t dd = static_cast<size_t>(head_dim) * 2;
    struct Span {
        const void *p;
        size_t n;
    };
    auto in = [&](const void *x, int64_t st, int n) {
        return Span{x, x == nullptr ? 0
                                    : (static_cast<size_t>(tokens) - 1) * static_cast<size_t>(st) * 2 +
                                          static_cast<size_t>(n) * dd};
    };
    const Span ins[3] = {in(Q, q_stride, n_q_heads), in(K, k_stride, kv_heads),
                         in(V, v_stride, kv_heads)};
    const Span outs[3] = {{Q_out, static_cast<size_t>(tokens) * n_q_heads * dd},
                          {K_out, static_cast<size_t>(tokens) * kv_heads * dd},
                          {V_out, V_out != nullptr ? static_cast<size_t>(tokens) * kv_heads * dd : 0}};
    const bool same[3] = {Q_out == Q && q_stride == static_cast<int64_t>(n_q_heads) * head_dim,
                          K_out == K && s == 1 && k_stride == static_cast<int64_t>(kv_heads) * head_dim,
                          V_out == V && s == 1 && v_stride == static_cast<int64_t>(kv_heads) * head_dim};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 3; ++i) {
            if (overlap(outs[o].p, outs[o].n, ins[i].p, ins[i].n) && !(o == i && same[o]))
                return fail(MLKV_ERR_INVALID_ARG, "an output overlaps an input");
            if (i < o && overlap(outs[o].p, outs[o].n, outs[i].p, outs[i].n))
                return fail(MLKV_ERR_INVALID_ARG, "two outputs overlap");
        }
    }
    NormRopeParams p;
    p.Q = static_cast<const __nv_bfloat16 *>(Q);
    p.K = static_cast<const __nv_bfloat16 *>(K);
    p.V = static_cast<const __nv_bfloat16 *>(V);
    p.q_stride = q_stride;
    p.k_stride = k_stride;
    p.v_stride = v_stride;
    p.q_gain = static_cast<const __nv_bfloat16 *>(q_gain);
    p.k_gain = static_cast<const __nv_bfloat16 *>(k_gain);
    p.cos = cos_table;
    p.sin = sin_table;
    p.positions = positions;
    p.q_out = static_cast<__nv_bfloat16 *>(Q_out);
    p.k_out = static_cast<__nv_bfloat16 *>(K_out);
    p.v_out = static_cast<__nv_bfloat16 *>(V_out);
    p.eps = eps;
    p.tokens = static_cast<int>(tokens);
    p.s = s;
    p.h = n_q_heads;
    p.g = kv_heads;
    p.heads = static_cast<int>(heads);
    p.rot = rot_dim;
    p.n_pos = n_pos;
    p.interleaved = interleaved != 0 ? 1 : 0;
    // Few tokens: one load a lane, so that the heads spread over the GPU.  Many: four, for the bytes
    // in flight and the table's reuse.
    const int hpi = 256 / head_dim;
    const long long loads = tokens * ((heads + hpi - 1) / hpi);
    const int U = loads >= 152LL * 64 * 4 ? 4 : 1;
    p.chunks = static_cast<int>((heads + static_cast<long long>(U) * hpi - 1) / (U * hpi));
    const long long blocks = (tokens * p.chunks + kNormThreads / 32 - 1) / (kNormThreads / 32);
    if (blocks > 0x7fffffffLL)
        return fail(MLKV_ERR_UNSUPPORTED, "%lld tokens of %lld heads exceed what one call takes",
                    tokens, heads);
    DeviceGuard guard(current_device());
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(kNormThreads);
    cfg.stream = static_cast<cudaStream_t>(cuda_stream);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    void *args[] = {&p};
    const void *fn = head_dim == 64 ? (U == 4 ? norm_fn<64, 4>() : norm_fn<64, 1>())
                                    : (U == 4 ? norm_fn<128, 4>() : norm_fn<128, 1>());
    const cudaError_t e = cudaLaunchKernelExC(&cfg, fn, args);
    return e == cudaSuccess ? MLKV_OK : fail_cuda(e, "qk_norm_rope launch");
}
