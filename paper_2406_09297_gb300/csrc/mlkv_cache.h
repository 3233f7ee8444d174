// The bf16 cache's handle, shared by the host side's translation units.  Internal; not part of the public ABI.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <vector>

#include "mlkv_host.h"
#include "mlkv_internal.h"

struct mlkv_cache {
    int l = 0, h = 0, d = 0, g = 0, G = 0, b = 0, max_seq = 0, m = 0;
    std::vector<int> owner, slot;
    int device = 0;
    int sm_count = 0;
    int l2_bytes = 0;
    int window_max = 0;
    size_t max_smem = 0;        // opt-in dynamic shared memory per block
    void *cache = nullptr;      // [m][2][b][g][max_seq][d] bf16
    size_t cache_bytes = 0;
    float *part_o = nullptr;    // [pieces][G][d]
    float *part_lse = nullptr;  // [pieces][G]
    unsigned *counters = nullptr;
    int *err = nullptr;
    int max_ctas = 0;           // capacity of the partial buffers beyond b*g pieces
    long long records = 0;      // partial records the scratch holds
    // options
    int tile_tokens = 0;
    int grid = 0;
    int l2_persist = 0;
    size_t persist_bytes = 0;   // the context's persisting-L2 set-aside while l2_persist is on
    size_t persist_prev = 0;    // the set-aside before l2_persist was switched on
    int l2_prefetch = 0;        // multi-layer step: prefetch the step's slots into L2 when they fit
    int step_kernel = 1;        // mlkv_decode_step: one multi-layer launch where it applies
    int last_step_kernel = 0;   // 1 if the most recent step ran as one multi-layer launch
    int last_seg_major = 0;     // 1 if that launch ranked its items segment-major
    int cluster = 1;            // allow the DSMEM cluster merge
    int pdl = 1;                // programmatic dependent launch
    int early_fetch = 1;        // per-layer step: later layers read Q and tiles before the wait
    int tc = 0;                 // 1: the tcgen05 kernel where a variant exists (slower here)
    int prefill_ready = 0;      // the prefill kernels' shared-memory limits are set (1 all, 2 windowed)
    int fused_ready = 0;        // the same for the fused-decode forms (bit 1 << form)
    int fused_deep = 1;         // fused decode: the deep one-tile form where one unit per SM
    // Context-chunk partials of the fused decode.  A buffer that was outgrown lives until the cache
    // is destroyed: recorded graphs, the caller's captures among them, hold its address.
    float *fused_part = nullptr;
    size_t fused_part_floats = 0;
    std::vector<float *> fused_outgrown;
    int step_fused = 1;         // mlkv_decode_step: the cross-layer fused form where it pays (1),
                                // wherever the map allows it (2), never (0)
    int last_step_fused = 0;    // 1 if the most recent step ran in that form
    int last_step_launches = 0;   // this library's launches in the most recent step
    int last_fused_kc = 0;      // key tiles per unit (chunk) of the most recent fused decode
    int fused_kc = 0;           // > 0: key tiles per unit of the fused decode, else planned
    // mlkv_decode_step's recorded graph and the arguments it was recorded for
    int step_graph = 2;         // 2: direct when one multi-layer launch, else record/replay
    cudaStream_t record_stream = nullptr;   // private stream the step graph is recorded on
    cudaGraphExec_t step_exec = nullptr;
    struct StepKey {
        const void *Q = nullptr, *K = nullptr, *V = nullptr;
        void *out = nullptr;
        std::vector<int> lens;
        int tile = -1, grid = -1, cluster = -1, pdl = -1, l2 = -1, tc = -1, pf = -1, sk = -1;
        int sg = -1;   // step_graph: a graph recorded under one mode is not replayed under another
        int ef = -1, sf = -1, fd = -1, fk = -1;
        bool operator==(const StepKey &o) const
        {
            return Q == o.Q && K == o.K && V == o.V && out == o.out && lens == o.lens &&
                   tile == o.tile && grid == o.grid && cluster == o.cluster && pdl == o.pdl &&
                   l2 == o.l2 && tc == o.tc && pf == o.pf && sk == o.sk && sg == o.sg &&
                   ef == o.ef && sf == o.sf && fd == o.fd && fk == o.fk;
        }
    } step_key, pending_key;   // recorded arguments; arguments seen once, not yet recorded
    int step_graph_replays = 0;
    // mlkv_decode_step_host: device staging of the step's inputs and outputs, its own graph
    void *stage = nullptr;     // Q [l][b][h][d], K, V [m][b][g][d], out [l][b][h][d]
    cudaGraphExec_t host_exec = nullptr;
    cudaStream_t side = nullptr;   // the copies that overlap the step's layers
    cudaEvent_t ev[2] = {nullptr, nullptr};   // fork, the later layers' queries in
    StepKey host_key, host_pending;
    // the most recent decode launch (read-only options, for tests and tuning)
    int last_grid = 0, last_tile = 0, last_cluster_k = 0, last_deferred = 0, last_tc = 0;
    int last_l2_prefetch = 0;
    // the most recent call behind shared prefixes: the form it took, and this library's launches (a store's apart)
    int last_prefix_form = 0, last_prefix_launches = 0;
    unsigned long_ready = 0;   // kernels of mlkv_long_host.cpp whose limits are set (a bit each)
    int piece_ctas = 0;        // resident CTAs of the piece kernel per SM
    // per-variant launch state
    struct Variant {
        const mlkv::DecodeVariant *v = nullptr;
        CUtensorMap tmap;        // boxes of tile_tokens positions
        CUtensorMap tmap_rows;   // boxes of 64 positions (a partly visible last tile)
        int ctas_per_sm = 0;
        int clusters[5] = {0, 0, 0, 0, 0};   // resident k-CTA clusters, k = 2, 4
    };
    std::vector<Variant> variants;
    std::vector<int> tile_start_scratch;
};

namespace mlkv {

// Makes c->fused_part hold `floats`; a buffer that was outgrown lives on (see mlkv_cache).
int grow_scratch(mlkv_cache *c, size_t floats, const char *what);
// The checks of a handle and a layer, and of the lengths of a cache's sequences.
int check_layer(const mlkv_cache *c, int layer);
int check_seq_lens(const mlkv_cache *c, const int *seq_lens);
// Whether two caches hold the same model's layers and heads, on one device.
int check_same_model(const mlkv_cache *c, const mlkv_cache *other, const char *what);
// The checks of a shared prefix's cache, of each sequence's prefix in it (-1: none) and of their lengths.
int check_prefix(const mlkv_cache *c, const mlkv_cache *prefix, const int *prefix_of, const int *prefix_lens);

// Forms of the calls behind shared prefixes (option "last_prefix_form").
enum : int {
    kFormNone = 0,
    kFormJoined = 1,    // each sequence's prefix and positions end to end
    kFormGroups = 2,    // a prefix for 16 heads at a time, in the suffixes' launch
    kFormKernel = 3,    // the prefix kernel, then the suffixes
    kFormBeside = 4,    // the prefix kernel and the suffixes side by side
    kFormPrompt = 5,    // prompts: the prefill's kernel (else their rows' form)
};

// Query rows of a decode over shared prefixes: row i attends to prefix[i]'s positions (-1: none) and then to the
// first len[i] of its sequence.  scattered: it is row q_row[i] of Q and out, of sequence seq[i]; else n is the
// cache's batch and every row its sequence's.
struct PrefixRows {
    int n, scattered, q_rows;   // q_rows: rows of Q
    uint16_t q_row[MLKV_MAX_BATCH], seq[MLKV_MAX_BATCH];
    int len[MLKV_MAX_BATCH], prefix[MLKV_MAX_BATCH];
};
// What a decode of a prompt's rows has to do besides.
struct PromptStep {
    double most_us;      // the decode is issued if it is estimated to take less,
    bool issued;         // which is told here, as is scratch that cannot be had: the prompt can do without
    int (*store)(const PromptStep &step, cudaStream_t stream);   // in front of the launches, behind every check
    mlkv_cache *c;       // the store's: K, V of s_max positions into the layer's slot, if they are to be stored
    int layer, s_max;
    const void *K, *V;
};
// Issues the decode, with everything checked and nothing queued on an error of a check.
int decode_rows(mlkv_cache *c, int layer, const mlkv_cache *prefix, const int *prefix_lens, const PrefixRows &rows,
                const void *Q, void *out, cudaStream_t stream, PromptStep *step = nullptr);

}  // namespace mlkv
