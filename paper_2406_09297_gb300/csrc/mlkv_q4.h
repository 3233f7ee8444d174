// The 4-bit KV cache: its layout and the interface between its host side (mlkv_q4_host.cpp) and its
// kernels (mlkv_q4.cu, mlkv_q4_decode.cu).  Internal; not part of the public ABI.
//
// Value.  32 consecutive channels of one position of one KV head share a scale, s = bf16(max |x| / 7);
// a channel is held as the whole number q in [-7, 7] nearest to x / s (halves away from zero), as sign
// and magnitude in 4 bits, and stands for q s.  A group with a NaN or an infinity holds NaN; one whose
// scale would be below 2^-126 holds zeros.
//
// Layout.  [m slots][b][g] rows, each a run of blocks of 16 positions, 18 D bytes a block: the codes
// of K (8 D), the codes of V (8 D), the scales of K (D), the scales of V (D).  Inside a block the codes
// lie as the lanes of a warp (lane = 4 gid + tig) want them for the A operand of mma.m16n8k16, a 32-bit
// word of 8 codes at a time.  A word as it is, rotated right by 4, shifted left by 8 and by 4, masked with
// 0x87008700, is its pairs j = 0 .. 3 of fp16 numbers, the sign in the sign bit and the magnitude m in
// bits 8 to 10: the top two mantissa bits and the lowest exponent bit, where subnormals and the first
// binade make one scale of m 2^-16.  (The masks, moved back, tile the word.  Left shifts go to the
// multiply-add pipe: the integer pipe, at half rate, is what bounds the unpacking.)
//   K, positions as rows: word (position, group, tig) holds the group's channels 8 tig + e, pair j =
//     e / 2, low half first.
//   V, channels as rows: word (position pair, group, gid) holds channels 4 gid + j of the group, pair j
//     the even position (low half) and the odd one (high half): their bits interleave in the word.
// A lane's words of one 16-byte load are its groups (D = 128), or its two groups of both halves of the
// block (D = 64).
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "mlkv_internal.h"

namespace mlkv {

constexpr int kQ4Group = 32;       // channels that share a scale
constexpr int kQ4Block = 16;       // positions of a block
constexpr int kQ4RowAlign = 64;    // a row's positions are rounded up to this

constexpr long long q4_row_bytes(int max_seq, int d)
{
    return (static_cast<long long>(max_seq) + kQ4RowAlign - 1) / kQ4RowAlign * (kQ4RowAlign / kQ4Block) *
           18LL * d;
}

template <int D>
struct Q4Layout {
    static constexpr int kGroups = D / kQ4Group;
    static constexpr int kBytes = 18 * D;          // of a block
    static constexpr int kV = 8 * D, kKs = 16 * D, kVs = 17 * D;
    // byte offsets inside a block of position r (0 .. 15)
    __host__ __device__ static constexpr int k_word(int r, int grp, int tig)
    {
        const int lane = (r & 7) * 4 + tig, hi = r >> 3;
        return 4 * (D == 128 ? (hi * 32 + lane) * 4 + grp : lane * 4 + hi * 2 + grp);
    }
    __host__ __device__ static constexpr int v_word(int r, int grp, int gid)
    {
        const int lane = gid * 4 + ((r & 7) >> 1), hi = r >> 3;
        return kV + 4 * (D == 128 ? (hi * 32 + lane) * 4 + grp : lane * 4 + hi * 2 + grp);
    }
    __host__ __device__ static constexpr int k_scale(int r, int grp)
    {
        return kKs + 2 * (r * kGroups + grp);
    }
    __host__ __device__ static constexpr int v_scale(int r, int grp)
    {
        return kVs + 2 * ((((((r & 7) >> 1) * 2 + (r >> 3)) * kGroups) + grp) * 2 + (r & 1));
    }
};

constexpr uint32_t kQ4Mask = 0x87008700u;
constexpr float kQ4Unit = 65536.f;   // what makes a magnitude whole
// The bits of half o of all pairs.
__host__ __device__ constexpr uint32_t q4_bits(int o) { return o ? 0xfff70008u : 0x0008fff7u; }

#ifdef __CUDACC__
// Pair j of a code word as fp16 in units of 2^-16.
__device__ __forceinline__ uint32_t q4_pair(uint32_t w, int j)
{
    const uint32_t x = j == 0 ? w : j == 1 ? __funnelshift_r(w, w, 4) : j == 2 ? w * 256u : w * 16u;
    return x & kQ4Mask;
}

// The word of four pairs (bits of kQ4Mask only).
__device__ __forceinline__ uint32_t q4_word(uint32_t p0, uint32_t p1, uint32_t p2, uint32_t p3)
{
    return p0 | __funnelshift_l(p1, p1, 4) | p2 >> 8 | p3 >> 4;
}
#endif

// Stores positions of K and V [b][g][len][D] (store) or of one new token [b][g][D] at seq_len - 1
// (append) into one slot.
struct Q4StoreParams {
    const __nv_bfloat16 *K, *V;
    uint8_t *slot;             // the slot's rows
    long long row_bytes;
    int b, g, len;             // len: positions [0, len) (store)
    int seq_len[MLKV_MAX_BATCH];   // append only
};
cudaError_t launch_q4_store(int d, const Q4StoreParams &p, cudaStream_t stream);
cudaError_t launch_q4_append(int d, const Q4StoreParams &p, cudaStream_t stream);

// Positions [start, start + len) of one slot as bf16 [b][g][len][D].
struct Q4ReadParams {
    __nv_bfloat16 *K, *V;
    const uint8_t *slot;
    long long row_bytes;
    int b, g, start, len;
};
cudaError_t launch_q4_read(int d, const Q4ReadParams &p, cudaStream_t stream);

struct Q4DecodeParams {
    const __nv_bfloat16 *Q;    // [b][h][D]
    __nv_bfloat16 *out;        // [b][h][D]
    const uint8_t *slot;
    long long row_bytes;
    float *part_o;             // [records][G][D]
    float *part_lse;           // [records][G]
    unsigned *counters;        // [b * g], zero between launches
    int *err;
    float scale_log2;          // log2(e) / sqrt(D)
    int b, h, g, G;
    int window, sinks;
    int num_tiles;
    // of the tiles: empty ones behind every segment's.  Runs of warps: empty_tiles, for the ends' cost; of
    // CTAs: as many as make its tiles a multiple of round_tiles, a run's (0: runs of warps)
    int empty_tiles, round_tiles;
    int uniform_len;           // the common length, or 0
    int deferred_merge;        // 1: combine_kernel merges the records
    int seq_len[MLKV_MAX_BATCH];
    int tile_start[MLKV_MAX_BATCH + 1];
};
// Positions per tile of the decode kernel, and its launch.
constexpr int q4_tile_tokens(int d) { return d == 128 ? 32 : 64; }
cudaError_t prepare_q4_decode(int d, int group, int *ctas_per_sm);
// Warps of a CTA, two CTAs an SM: what the accumulators of 8 or 16 heads leave registers for.  Measured, us:
// 32 sequences of 16384, groups of 16 heads of 128, with 4 / 5 / 6 / 8 warps 51.4 / 83.4 / 79.7 / 107.4; 64 of
// 16384, groups of 12 heads of 64, 27.9 / 32.7 / 28.5 / 39.5.
constexpr int q4_warps(int d, int group) { return group <= 8 ? 8 : d == 64 ? 6 : 4; }
// Records of warps' runs up to which the warp that finishes a segment merges them (else a launch of its own).
constexpr int kQ4InlineMergePieces = 16;
// warp_runs: P = grid x warps runs of tiles, a warp each; else P = grid, a CTA each (see the kernel).
cudaError_t launch_q4_decode(int d, int grid, bool warp_runs, const Q4DecodeParams &p,
                             cudaStream_t stream);

}  // namespace mlkv
