// Internal interface of the operators for long caches: decode over pieces of a cache (a shared prefix's
// suffixes, listed blocks, or all positions with their weights), blocks' bounds and their selection,
// eviction.  Not part of the public ABI.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "mlkv_internal.h"

namespace mlkv {

// Positions of a block, of a tile of the piece kernel, and rows of the cache's 64-position tensor map.
constexpr int kBlock = MLKV_BLOCK;

// What a piece launch attends to.
enum : int {
    kPieceSuffix = 0,   // positions [0, seq_len), merged with a shared prefix's records
    kPieceBlocks = 1,   // the blocks listed for every (sequence, KV head)
    kPieceWeights = 2,  // positions [0, seq_len); every score is stored, the merge left to weights_kernel
    kPieceJoined = 3,   // a prefix's positions, read for every sequence apart, and then [0, seq_len)
    kPieceGroups = 4,   // kPieceSuffix with units in front, each a chunk of a prefix's positions for a few sequences
};

constexpr int kPieceMaxUnits = 1024;

// Decode attention of one layer in pieces: a segment (sequence, KV head) of nt tiles of 64 positions is cut
// into pieces of `tiles` tiles, a CTA each.  Passed by value, each mode its part (PieceArgs): 16 KB more of them cost
// the host 0.2 us a launch.
struct PieceBase {
    const __nv_bfloat16 *Q;   // [b][h][D]
    __nv_bfloat16 *out;       // [b][h][D]
    float *part_o;            // [pieces][G][D]  normalised outputs of pieces
    float *part_lse;          // [pieces][G]     log2 of their sums, -inf for an empty piece
    unsigned *counters;       // [b*g]           pieces finished per segment; zero between launches
    int *err;
    float scale_log2;         // log2(e) / sqrt(D)
    int b, h, g, G, slot;     // b: sequences of the cache
    // The query rows: decode has one a sequence, in their order; a prompt's tokens are rows of their own
    // (scattered: row i is row q_row[i] of Q and out, of sequence seq[i]).
    int n, scattered;
    int tiles;                // of a piece
    // kPieceSuffix: records of the shared prefix, [place][g][pre_chunks][G][D] and [place][g][pre_chunks][G]
    // with place = pre_place[beta] (below); 0 chunks: none
    const float *pre_o, *pre_lse;
    int pre_chunks;
    int early;                // the stream's previous kernel is this call's prefix kernel, which writes
                              // neither Q nor the cache and has itself waited for all before it: Q and
                              // the tiles are read before the dependency wait
    int defer;                // every piece writes its record, launch_merge_pieces merges them: many records, or
                              // pieces that run beside a prefix kernel, for which then nothing but that waits
    // kPieceBlocks: block numbers [b][g][n_blocks]; others than those of visible positions are passed over
    const int *blocks;
    int n_blocks;
    // kPieceWeights: scores times log2(e) / sqrt(D), [b][h][score_stride]
    float *scores;
    long long score_stride;
    int ordered;                          // rows are laid out as order lists them, the longest first; 0: as they are
    uint16_t order[MLKV_MAX_BATCH];
    int first[MLKV_MAX_BATCH + 1];        // first piece of the i-th row in that order (KV head after KV head inside)
    int seq_len[MLKV_MAX_BATCH];          // positions that a row sees
};
// What runs over prefixes; arrays by row.
struct PiecePrefix : PieceBase {
    int prefix_b;                         // kPieceJoined, kPieceGroups: sequences of the prefix cache
    union {
        struct {
            uint16_t q_row[MLKV_MAX_BATCH], seq[MLKV_MAX_BATCH];   // scattered
        };
        int prefix_len[MLKV_MAX_BATCH];   // kPieceGroups: of the prefix cache's sequences
    };
    uint16_t pre_place[MLKV_MAX_BATCH];   // kPieceSuffix: its place in the prefix's records;
                                          // kPieceJoined: its prefix's number
    union {
        struct {
            uint16_t pre_n[MLKV_MAX_BATCH];         // kPieceSuffix: those records' number
            uint16_t place_row[MLKV_MAX_BATCH];     // kPieceGroups: the row at a place
        };
        int pre_len[MLKV_MAX_BATCH];      // kPieceJoined: positions of its prefix, 0: none
    };
};
// And what has units.
struct PieceParams : PiecePrefix {
    // kPieceGroups: units, the launch's first CTAs: unit_tiles tiles from unit_tiles * chunk on of a prefix, for the
    // heads of KV head j of up to 16 / G rows from a place on.
    int n_units, unit_tiles;
    uint32_t units[kPieceMaxUnits];       // prefix | chunk << 10 | j << 18 | (rows - 1) << 26
    uint16_t unit_place[kPieceMaxUnits];
};
static_assert(sizeof(PieceParams) + 2 * sizeof(CUtensorMap) < 32764, "kernel parameters");
template <int kMode>
using PieceArgs = std::conditional_t<kMode == kPieceGroups, PieceParams,
                                     std::conditional_t<kMode == kPieceSuffix || kMode == kPieceJoined, PiecePrefix,
                                                        PieceBase>>;

// Tiles of a segment.
template <int kMode>
__host__ __device__ inline int piece_tiles(const PieceArgs<kMode> &p, int beta)
{
    if constexpr (kMode == kPieceBlocks)
        return p.n_blocks;
    const int own = static_cast<int>((static_cast<unsigned>(p.seq_len[beta]) + kBlock - 1) / kBlock);
    if constexpr (kMode == kPieceJoined)
        return static_cast<int>((static_cast<unsigned>(p.pre_len[beta]) + kBlock - 1) / kBlock) + own;
    return own;
}
// Most records (pieces and a prefix's) that a segment's merge holds the weights of.
int piece_max_records(int head_dim, int group);
int piece_stages(int head_dim);   // tiles of a piece that are worked on at a time
cudaError_t prepare_pieces(int head_dim, int group, int mode, int *ctas_per_sm);
// tmap_prefix: the prefix cache's (kPieceJoined; else not read).
cudaError_t launch_pieces(int head_dim, int mode, const CUtensorMap *tmap, const CUtensorMap *tmap_prefix,
                          const PieceParams &p, cudaStream_t stream);

// The merge of a deferred launch's segments, of `most` records at most.
cudaError_t launch_merge_pieces(int head_dim, int mode, const PieceParams &p, int most, cudaStream_t stream);

// Most records of a segment that launch_merge_pieces and launch_weights take (the weights of two heads' records in
// 48 KB of shared memory).
constexpr int kDeferMaxRecords = 4096;

// The merge of a kPieceWeights launch's pieces, and what every position got: out, and
// weights_out[beta][j][u] = weights_in[beta][j][u] + sum over the heads of the group.
struct WeightsParams {
    const float *weights_in;   // [b][g][max_seq] or nullptr: zeros
    float *weights_out;        // [b][g][max_seq]
    int max_seq;
    int chunk;                 // positions of a CTA
    int merge_ctas, wide;      // of a segment: CTAs that merge its records, many of them (plan_weights)
    int ctas;                  // of a segment: those, then those of its positions
};
void plan_weights(int head_dim, int group, int most, WeightsParams *w);
cudaError_t launch_weights(int head_dim, const PieceParams &p, const WeightsParams &w, int most,
                           cudaStream_t stream);

struct BoundsParams {
    const __nv_bfloat16 *K;    // [b][g][max_seq][D], the slot's keys
    int8_t *bounds;            // [b][g][n_blocks][2][D]
    float *scales;             // [b][g][n_blocks]
    int b, g, max_seq, n_blocks;
    int seq_len[MLKV_MAX_BATCH];
    int first[MLKV_MAX_BATCH]; // first position that is new
    int per_cta;                     // blocks of a CTA
    int start[MLKV_MAX_BATCH + 1];   // first CTA of a sequence
};
int bounds_per_cta(long long blocks, int sm_count);
cudaError_t launch_bounds(int head_dim, const BoundsParams &p, cudaStream_t stream);

struct SelectParams {
    const __nv_bfloat16 *Q;    // [b][h][D]
    const int8_t *bounds;
    const float *scales;
    int *blocks;               // [b][g][n_select]
    int b, h, g, G, n_blocks, n_select, n_first, n_last;
    int seq_len[MLKV_MAX_BATCH];
};
// Most blocks of a sequence that a selection handles.
int select_max_blocks();
cudaError_t prepare_select(int head_dim);
cudaError_t launch_select(int head_dim, const SelectParams &p, int max_blocks, cudaStream_t stream);

struct EvictParams {
    const __nv_bfloat16 *src;  // the slots: [2][b][g][src_seq][D]
    __nv_bfloat16 *dst;        // [2][b][g][dst_seq][D]
    const float *weights_in;   // [b][g][src_seq]
    float *weights_out;        // [b][g][dst_seq]
    int *kept;                 // [b][g][k_max]
    unsigned *flags;           // [b][g][units] units whose rows have been read, then the ticket
    int *err;
    int b, g, src_seq, dst_seq, k_max, recent;
    int in_place;              // the slots or the weights are the same memory
    int same;                  // both are: rows that stay where they are need no store
    int units;                 // of a segment: ceil(rows / rows of a unit), and one for the tail
    int rows;                  // that stay of a segment, at most
    int seq_len[MLKV_MAX_BATCH];
    int keep[MLKV_MAX_BATCH];
};
// Units of a segment of k_max kept positions; flags that a launch needs for `segments` of them.
int evict_units(int head_dim, int k_max);
inline size_t evict_flags(long long segments, int units) { return static_cast<size_t>(segments) * units + 1; }
cudaError_t prepare_evict();
cudaError_t launch_evict(int head_dim, const EvictParams &p, int max_len, int sm_count, cudaStream_t stream);

}  // namespace mlkv
