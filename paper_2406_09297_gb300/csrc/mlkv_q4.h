// The 4-bit KV cache: its layout and the interface between its host side (mlkv_q4_host.cpp) and its
// kernels (mlkv_q4.cu, mlkv_q4_decode.cu).  Internal; not part of the public ABI.
//
// Value.  32 consecutive channels of one position of one KV head share a scale, s = bf16(max |x| / 7);
// a channel is held as the whole number q in [-7, 7] nearest to x / s (halves away from zero), code
// q + 8, and stands for q s.  A group with a NaN or an infinity holds NaN; one whose scale would be
// below 2^-126 holds zeros.
//
// Layout.  [m slots][b][g] rows, each a run of blocks of 16 positions, 18 D bytes a block: the codes
// of K (8 D), the codes of V (8 D), the scales of K (D), the scales of V (D).  Inside a block the codes
// lie as the lanes of a warp want them for mma.m16n8k16, lane = 4 gid + tig, one 32-bit word a lane
// holding four bf16 pairs once its nibbles i and i + 4 (bits 4 i and 16 + 4 i) are set apart:
//   K, positions as the rows of A (gid, gid + 8): word (position, group, tig) holds the group's
//     channels 8 tig .. 8 tig + 7, channel 8 tig + e in nibble e / 2 of half e % 2.
//   V, channels as the rows of A, positions along k: word (position pair, group, gid) holds channels
//     4 gid .. 4 gid + 3 of the group, channel 4 gid + i in nibble i, of the even position in the low
//     half and of the odd one in the high half.  So one position owns whole 16-bit halves, and storing
//     it reads nothing.
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
    int uniform_len;           // the common length, or 0
    int deferred_merge;        // 1: combine_kernel merges the records
    int seq_len[MLKV_MAX_BATCH];
    int tile_start[MLKV_MAX_BATCH + 1];
};
// Positions per tile of the decode kernel, and its launch.
constexpr int q4_tile_tokens(int d) { return d == 128 ? 32 : 64; }
cudaError_t prepare_q4_decode(int d, int group, int *ctas_per_sm);
cudaError_t launch_q4_decode(int d, int grid, const Q4DecodeParams &p, cudaStream_t stream);

}  // namespace mlkv
