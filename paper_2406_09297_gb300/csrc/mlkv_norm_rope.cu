// Queries, keys and values of a projection made ready for the cache's calls (mlkv_qk_norm_rope): RMS
// norm of every query and key head, rotary position encoding in the same pass, values moved along.
//
//   y = x / sqrt(mean(x^2) + eps) * gain           per head, over its D channels
//   (a, b) -> (a cos - b sin, b cos + a sin)       on the first rot channels, (a, b) = channels i and
//                                                  i + rot/2, or 2i and 2i + 1 (interleaved)
//
// In fp32, rounded once, to bf16.  Every channel is read once and written once; at 4 bytes a channel HBM
// leaves ~12 instructions for the 8 channels of a 16-byte load, so the instructions are kept few: a lane
// holds 16 channels of a head, two pieces of 8 that are each other's rotation partners, and D / 16 lanes
// a head, so that only the sum of squares crosses lanes; gain and rotation are one pair of factors a
// channel, made once per token:
//   a' = r (a (g_a cos) - b (g_b sin)),  b' = r (b (g_b cos) + a (g_a sin)),  r = 1 / sqrt(...)
// A block's warps take heads of one kind (queries, keys or values), whose addresses are then uniform: of one
// token or several, up to 512 / D heads at a time, two (D = 64: three) such loads in flight.
//
// Measured on GB300: 16,004 tokens of 32 + 8 + 8 heads of 128 in 63.3 us, 6.2 TB/s of 6.8 (97.6 with the
// partner channels fetched from other lanes and factors made a head); 32,000 of 12 + 4 + 4 heads of 64 in
// 29.8 us, 5.6 TB/s.  Heads of 64 are bound by latency (a token's position, then its factors): several tokens
// a warp, few enough heads of each at a time that they take three loads and divide evenly (39.3 us with
// whole tokens a warp, the last load half empty), five blocks an SM for their registers (six with two
// loads 30.4, four 32.7).  A batch's single tokens are bound by the caller: 7.0 us of Python and launch.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <cmath>

#include "mlkv_host.h"

#include "mlkv_device.cuh"

namespace mlkv {
namespace {

struct NormRopeParams {
    // by kind: queries, keys, values
    const __nv_bfloat16 *in[3];                // token rows of heads, in_stride elements apart
    long long in_stride[3];
    const __nv_bfloat16 *gain[2];              // [D] or null
    __nv_bfloat16 *out[3];
    long long out_seq[3], out_token[3], out_head[3];   // elements: a sequence, token, head further
    int heads[3];
    int wide[3];                               // heads of a token that a warp holds at a time (a power of
                                               // two; 512 / D: one token a warp)
    int parts[3];                              // warps that share a token's heads
    unsigned first_block[3];                   // of the kind's blocks, part by part
    const float *cos, *sin;                    // [n_pos][rot / 2]
    const int *positions;                      // [tokens]
    float eps;
    int tokens, s, rot, n_pos;
    int per_block;                             // heads of a block, a multiple of 512 / D
};

constexpr int kNormThreads = 128;
// Loads of a lane in flight.
__host__ __device__ constexpr int norm_loads(int d) { return d == 64 ? 3 : 2; }

// kInter: pairs are neighbouring channels.
template <int D, bool kInter>
__global__ void __launch_bounds__(kNormThreads, D == 64 ? 5 : 6)
    norm_rope_kernel(const __grid_constant__ NormRopeParams p)
{
    constexpr int LPH = D / 16;       // lanes per head
    constexpr int HPI = 32 / LPH;     // heads a warp holds at a time
    constexpr int U = norm_loads(D);
    grid_dependency_wait();
    grid_dependents_launch();
    const int kind = blockIdx.x < p.first_block[1] ? 0 : blockIdx.x < p.first_block[2] ? 1 : 2;
    const int lane = threadIdx.x & 31;
    const int sel = lane / LPH, wide = p.wide[kind], parts = p.parts[kind];
    // heads from a lane's load to its next (of 128 channels, fewer than HPI heads are one load)
    const int step = D == 64 ? wide : HPI;
    const unsigned block = (blockIdx.x - p.first_block[kind]) / parts;
    const int part = static_cast<int>(blockIdx.x - p.first_block[kind] - block * parts);
    // this lane's token; past the last one there is nothing to do, but the warp's shuffles need it
    const long long token_at =
        (static_cast<long long>(block) * (kNormThreads / 32) + (threadIdx.x >> 5)) * (HPI / wide) +
        sel / wide;
    const bool live = token_at < p.tokens;
    const int token = live ? static_cast<int>(token_at) : p.tokens - 1;
    // This lane's pieces of 8 channels: rotation partners, or (past the rotated ones) neighbours.
    const int c = lane % LPH;
    const int hp = p.rot / 16;        // pieces in half the rotated channels
    const bool rotates = c < hp;
    const int pa = kInter ? 16 * c : rotates ? 8 * c : 8 * (2 * hp + 2 * (c - hp));
    const int pb = kInter || !rotates ? pa + 8 : 8 * (c + hp);
    // its heads: from head0 on, `step` apart, below head1; no lane of the warp has any from `stop` on
    const int first = part * p.per_block, stop = min(p.heads[kind], first + p.per_block);
    const int head0 = first + sel % wide, head1 = live ? stop : 0;
    const int beta = token / p.s;
    const __nv_bfloat16 *src =
        p.in[kind] + token * p.in_stride[kind] + static_cast<long long>(head0) * D;
    __nv_bfloat16 *dst = p.out[kind] + beta * p.out_seq[kind] +
                         (token - beta * p.s) * p.out_token[kind] + head0 * p.out_head[kind];
    const int d_ab = pb - pa;
    src += pa;
    dst += pa;
    const long long out_step = step * p.out_head[kind];
    auto read = [&](uint4 (&a)[U], uint4 (&b)[U], int head) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (head + u * step < head1) {
                a[u] = *reinterpret_cast<const uint4 *>(src + u * step * D);
                b[u] = *reinterpret_cast<const uint4 *>(src + u * step * D + d_ab);
            }
        src += U * step * D;
    };
    uint4 xa[U], xb[U];
    if (kind == 2) {   // values only move
        for (int h0 = first, head = head0; h0 < stop; h0 += U * step, head += U * step) {
            read(xa, xb, head);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (head + u * step < head1) {
                    *reinterpret_cast<uint4 *>(dst) = xa[u];
                    *reinterpret_cast<uint4 *>(dst + d_ab) = xb[u];
                }
                dst += out_step;
            }
        }
        return;
    }
    read(xa, xb, head0);
    auto unpack = [](const uint4 &v, float (&f)[8]) {
        const uint32_t r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = bf16_lo(r[i]);
            f[2 * i + 1] = bf16_hi(r[i]);
        }
    };
    auto pack = [](const float (&f)[8]) {
        return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                          pack_bf16x2(f[6], f[7]));
    };
    // The factors of the lane's 8 pairs (elements i of both pieces, or, interleaved, neighbours: pairs
    // 0 .. 3 in piece a): gains times cos and sin, of the pairs' first and second elements.
    float ac[8], as[8], bc[8], bs[8];
    {
        float cs[8], sn[8], ga[8], gb[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            cs[i] = ga[i] = gb[i] = 1.f;
            sn[i] = 0.f;
        }
        const __nv_bfloat16 *gain = p.gain[kind];
        if (gain != nullptr) {
            unpack(*reinterpret_cast<const uint4 *>(gain + pa), ga);
            unpack(*reinterpret_cast<const uint4 *>(gain + pb), gb);
        }
        if (kInter ? 16 * c < p.rot : rotates) {
            const int pos = p.positions[token];
            if (pos >= 0 && pos < p.n_pos) {
                const size_t at = static_cast<size_t>(pos) * (p.rot / 2) + 8 * c;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const float4 a = *reinterpret_cast<const float4 *>(p.cos + at + 4 * q);
                    const float4 b = *reinterpret_cast<const float4 *>(p.sin + at + 4 * q);
                    cs[4 * q] = a.x;
                    cs[4 * q + 1] = a.y;
                    cs[4 * q + 2] = a.z;
                    cs[4 * q + 3] = a.w;
                    sn[4 * q] = b.x;
                    sn[4 * q + 1] = b.y;
                    sn[4 * q + 2] = b.z;
                    sn[4 * q + 3] = b.w;
                }
            } else {
                // outside the table: the rotated channels say so
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    cs[i] = __int_as_float(0x7fffffff);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float g0 = kInter ? (i < 4 ? ga[2 * i & 7] : gb[2 * i & 7]) : ga[i];
            const float g1 = kInter ? (i < 4 ? ga[(2 * i + 1) & 7] : gb[(2 * i + 1) & 7]) : gb[i];
            ac[i] = g0 * cs[i];
            as[i] = g0 * sn[i];
            bc[i] = g1 * cs[i];
            bs[i] = g1 * sn[i];
        }
    }
    for (int h0 = first, head = head0;;) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (h0 + u * step >= stop)
                break;
            float a[8], b[8], oa[8], ob[8];
            unpack(xa[u], a);
            unpack(xb[u], b);
            float s0 = 0.f, s1 = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s0 = fmaf(a[i], a[i], s0);
                s1 = fmaf(b[i], b[i], s1);
            }
            float ss = s0 + s1;
#pragma unroll
            for (int m = 1; m < LPH; m <<= 1)
                ss += __shfl_xor_sync(0xffffffffu, ss, m);
            const float r = rsqrtf(ss * (1.f / D) + p.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // pair i: x its first element, y its second
                const float x = kInter ? (i < 4 ? a[2 * i & 7] : b[2 * i & 7]) : a[i];
                const float y = kInter ? (i < 4 ? a[(2 * i + 1) & 7] : b[(2 * i + 1) & 7]) : b[i];
                const float x1 = r * fmaf(x, ac[i], -y * bs[i]), y1 = r * fmaf(y, bc[i], x * as[i]);
                if (kInter) {
                    (i < 4 ? oa : ob)[2 * i & 7] = x1;
                    (i < 4 ? oa : ob)[(2 * i + 1) & 7] = y1;
                } else {
                    oa[i] = x1;
                    ob[i] = y1;
                }
            }
            if (head + u * step < head1) {
                *reinterpret_cast<uint4 *>(dst) = pack(oa);
                *reinterpret_cast<uint4 *>(dst + d_ab) = pack(ob);
            }
            dst += out_step;
        }
        h0 += U * step;
        head += U * step;
        if (h0 >= stop)
            break;
        read(xa, xb, head);
    }
}

template <int D>
const void *norm_fn(bool interleaved)
{
    return interleaved ? reinterpret_cast<const void *>(&norm_rope_kernel<D, true>)
                       : reinterpret_cast<const void *>(&norm_rope_kernel<D, false>);
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
    if (Q == nullptr || Q_out == nullptr)
        return fail(MLKV_ERR_INVALID_ARG, "Q and Q_out must be non-NULL");
    if ((K == nullptr) != (K_out == nullptr) || (V == nullptr) != (V_out == nullptr))
        return fail(MLKV_ERR_INVALID_ARG, "K and K_out, V and V_out: both given or both NULL");
    if (K == nullptr && V != nullptr)
        return fail(MLKV_ERR_INVALID_ARG, "V without K");
    if (K == nullptr)
        kv_heads = 0;
    if (batch < 1 || s < 1 || n_q_heads < 1 || kv_heads < (K != nullptr))
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
    for (const int64_t st : {q_stride, k_stride, v_stride})   // addresses stay below 2^62
        if (st > (1LL << 60) / tokens)
            return fail(MLKV_ERR_UNSUPPORTED, "a token stride of %lld elements exceeds what one call takes",
                        static_cast<long long>(st));
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
                          {K_out, K_out != nullptr ? static_cast<size_t>(tokens) * kv_heads * dd : 0},
                          {V_out, V_out != nullptr ? static_cast<size_t>(tokens) * kv_heads * dd : 0}};
    auto dense = [&](int64_t st, int n) { return tokens == 1 || st == static_cast<int64_t>(n) * head_dim; };
    const bool same[3] = {Q_out == Q && dense(q_stride, n_q_heads),
                          K_out == K && s == 1 && dense(k_stride, kv_heads),
                          V_out == V && s == 1 && dense(v_stride, kv_heads)};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 3; ++i) {
            if (overlap(outs[o].p, outs[o].n, ins[i].p, ins[i].n) && !(o == i && same[o]))
                return fail(MLKV_ERR_INVALID_ARG, "an output overlaps an input");
            if (i < o && overlap(outs[o].p, outs[o].n, outs[i].p, outs[i].n))
                return fail(MLKV_ERR_INVALID_ARG, "two outputs overlap");
        }
    }
    NormRopeParams p;
    const void *in_ptr[3] = {Q, K, V};
    void *out_ptr[3] = {Q_out, K_out, V_out};
    const int64_t in_stride[3] = {q_stride, k_stride, v_stride};
    const long long d = head_dim;
    for (int k = 0; k < 3; ++k) {
        p.in[k] = static_cast<const __nv_bfloat16 *>(in_ptr[k]);
        p.in_stride[k] = in_stride[k];
        p.out[k] = static_cast<__nv_bfloat16 *>(out_ptr[k]);
        p.heads[k] = k == 0 ? n_q_heads : kv_heads;
        p.out_seq[k] = static_cast<long long>(s) * p.heads[k] * d;
        p.out_token[k] = k == 0 ? n_q_heads * d : d;
        p.out_head[k] = k == 0 ? d : s * d;
    }
    p.gain[0] = static_cast<const __nv_bfloat16 *>(q_gain);
    p.gain[1] = static_cast<const __nv_bfloat16 *>(k_gain);
    p.cos = cos_table;
    p.sin = sin_table;
    p.positions = positions;
    p.eps = eps;
    p.tokens = static_cast<int>(tokens);
    p.s = s;
    p.rot = rot_dim;
    p.n_pos = n_pos;
    // Few tokens: a load a warp, so that the heads spread over the GPU.  Many: all of a kind's heads, for
    // the factors' reuse.
    const int hpi = 512 / head_dim;
    const long long loads = tokens * ((heads + hpi - 1) / hpi);
    const bool many = loads >= 152LL * 64;
    p.per_block = many ? 16 * hpi : hpi;
    long long blocks = 0;
    for (int k = 0; k < 3; ++k) {
        p.wide[k] = 1;
        // many tokens, 64 channels a head: a divisor of the heads that makes three loads of them or more
        while (p.wide[k] < hpi && p.wide[k] < p.heads[k] &&
               !(many && head_dim == 64 &&
                 (p.heads[k] % (2 * p.wide[k]) != 0 || p.heads[k] < 6 * p.wide[k])))
            p.wide[k] *= 2;
        p.parts[k] = (p.heads[k] + p.per_block - 1) / p.per_block;
        p.first_block[k] = static_cast<unsigned>(blocks);
        const long long a_block = kNormThreads / 32 * (hpi / p.wide[k]);
        if (in_ptr[k] != nullptr)
            blocks += (tokens + a_block - 1) / a_block * p.parts[k];
        if (blocks > 0x7fffffffLL)
            return fail(MLKV_ERR_UNSUPPORTED, "%lld tokens of %lld heads exceed what one call takes",
                        tokens, heads);
    }
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
    const void *fn = head_dim == 64 ? norm_fn<64>(interleaved != 0) : norm_fn<128>(interleaved != 0);
    const cudaError_t e = cudaLaunchKernelExC(&cfg, fn, args);
    return e == cudaSuccess ? MLKV_OK : fail_cuda(e, "qk_norm_rope launch");
}

extern "C" int mlkv_qk_norm_rope_struct(const mlkv_qk_norm_rope_args *a)
{
    if (a == nullptr)
        return mlkv::fail(MLKV_ERR_INVALID_ARG, "args is NULL");
    return mlkv_qk_norm_rope(a->Q, a->K, a->V, a->q_stride, a->k_stride, a->v_stride, a->q_gain,
                             a->k_gain, a->cos_table, a->sin_table, a->n_pos, a->rot_dim,
                             a->interleaved, a->positions, a->eps, a->batch, a->s, a->n_q_heads,
                             a->kv_heads, a->head_dim, a->Q_out, a->K_out, a->V_out, a->cuda_stream);
}
