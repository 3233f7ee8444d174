// Host side of the 4-bit KV cache: argument checks, allocation and the mlkv_q4_* calls of mlkv.h.
//
// The cache of an MLKV model's m owner layers (arXiv 2406.09297, Sec. 3) as one allocation of
// [m][b][g] rows of blocks (mlkv_q4.h).  The decode kernel's tiles are dealt out here (deal); it shares
// the bf16 decode kernel's merge of many records (combine_kernel).
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "mlkv_host.h"
#include "mlkv_q4.h"

using mlkv::aligned16;
using mlkv::DeviceGuard;
using mlkv::fail;
using mlkv::fail_cuda;
using mlkv::overlap;

struct mlkv_q4cache {
    int l = 0, h = 0, d = 0, g = 0, G = 0, b = 0, max_seq = 0, m = 0;
    std::vector<int> owner, slot;
    int device = 0;
    int sm_count = 0;
    int ctas_per_sm = 0;
    uint8_t *cache = nullptr;   // [m][b][g] rows
    long long row_bytes = 0;
    size_t cache_bytes = 0;
    float *part_o = nullptr;    // [records][G][d]
    float *part_lse = nullptr;  // [records][G]
    unsigned *counters = nullptr;
    int *err = nullptr;
};

namespace {

void free_all(mlkv_q4cache *c)
{
    cudaFree(c->cache);
    cudaFree(c->part_o);
    cudaFree(c->part_lse);
    cudaFree(c->counters);
    cudaFree(c->err);
}

int check_layer(const mlkv_q4cache *c, int layer)
{
    if (c == nullptr)
        return fail(MLKV_ERR_INVALID_ARG, "null cache handle");
    if (layer < 0 || layer >= c->l)
        return fail(MLKV_ERR_INVALID_ARG, "layer %d outside [0, %d)", layer, c->l);
    return MLKV_OK;
}

int check_lens(const mlkv_q4cache *c, const int *seq_lens)
{
    if (seq_lens == nullptr)
        return fail(MLKV_ERR_INVALID_ARG, "seq_lens is NULL");
    for (int beta = 0; beta < c->b; ++beta)
        if (seq_lens[beta] < 1 || seq_lens[beta] > c->max_seq)
            return fail(MLKV_ERR_RANGE, "seq_lens[%d] = %d outside [1, %d]", beta, seq_lens[beta],
                        c->max_seq);
    return MLKV_OK;
}

// A prompt's keys and values, which kernels read where they lie: in memory of the cache's device.  (Another
// GPU's may not be mapped here, the host's may not be readable by kernels.)
int check_prompt_kv(const mlkv_q4cache *c, const void *K, const void *V)
{
    for (const void *x : {K, V}) {
        if (x == nullptr || !aligned16(x))
            return fail(MLKV_ERR_INVALID_ARG, "K and V must be non-NULL and 16-byte aligned");
        cudaPointerAttributes at;
        const cudaError_t e = cudaPointerGetAttributes(&at, x);
        if (e != cudaSuccess)
            cudaGetLastError();
        if (e != cudaSuccess || !((at.type == cudaMemoryTypeDevice && at.device == c->device) ||
                                  at.type == cudaMemoryTypeManaged))
            return fail(MLKV_ERR_INVALID_ARG, "K and V must lie in the memory of the cache's device");
    }
    return MLKV_OK;
}

uint8_t *slot_base(const mlkv_q4cache *c, int layer)
{
    return c->cache + c->cache_bytes / c->m * c->slot[layer];
}

int store(mlkv_q4cache *c, int layer, const void *K, const void *V, int len, const int *seq_lens,
          cudaStream_t stream)
{
    static thread_local mlkv::Q4StoreParams p;
    p.K = static_cast<const __nv_bfloat16 *>(K);
    p.V = static_cast<const __nv_bfloat16 *>(V);
    p.slot = slot_base(c, layer);
    p.row_bytes = c->row_bytes;
    p.b = c->b;
    p.g = c->g;
    p.len = len;
    if (seq_lens != nullptr)
        std::memcpy(p.seq_len, seq_lens, sizeof(int) * c->b);
    const cudaError_t e = seq_lens != nullptr ? mlkv::launch_q4_append(c->d, p, stream)
                                              : mlkv::launch_q4_store(c->d, p, stream);
    return e == cudaSuccess ? MLKV_OK : fail_cuda(e, "4-bit store launch");
}

constexpr int kEmpty = 3;   // runs of warps: empty tiles behind a segment

// Runs of at least `run` tiles that a segment of nt and the empty ones meets, at most.
long long warp_pieces(int nt, long long run) { return (nt + kEmpty - 2 + run) / run + 1; }

// Estimated us of merging S segments' records of CTAs, up to `pieces` each: by the CTA that finishes a
// segment, in round trips to L2 (8 records of four columns a thread), or by a launch of a CTA for every row.
// Measured, us, the first / the second: one sequence of 8192, 8 KV heads of 128, 4 query heads each, 16
// records 8.7 / 7.8, 32 records 9.6 / 8.0; 4 sequences of 4000, 2 KV heads, 16 query heads each, 16 records
// 12.5 / 9.5, 64 of them, 2 records 30.0 / 36.9.
struct Q4Merge {
    float us;
    bool deferred;
};
Q4Merge merge_of(const mlkv_q4cache *c, long long S, long long pieces)
{
    if (pieces <= 1)
        return {0.f, false};
    const int at_once = 4 * 32 * mlkv::q4_warps(c->d, c->G);
    const float here = 1.f + 0.9f * ((c->G * c->d + at_once - 1) / at_once) * ((pieces + 7) / 8);
    const float apart = (c->G <= 8 || c->d == 64 ? 2.4f : 4.2f) + 0.0034f * S * c->G;
    return {std::min(here, apart), apart < here};
}

// How a launch's tiles are dealt out (see mlkv_q4_decode_attention).
struct Q4Deal {
    int turns;       // of a CTA's warps per run; 0: a run per warp
    float us;        // estimated
};

// S segments of at most nt_max tiles, `sum` of them in all (warp_tiles with the empty ones); same: of one
// number of tiles.  The least of the estimated times, whose terms are fits to 137 calls, even and uneven: 4 to
// 512 sequences of 64 to 4000 positions, 2 of 30000 and 3 of 60000.  (Fitted to a kernel whose tiles took 8%
// less; the split taken was measured again against every other since: at most 6% behind the best in 129 of
// them, at most 14% in the rest.  Outside, the terms are extrapolated: one sequence of 131072, 12 heads of 64,
// 11.4 us; 8 of 65536, 8 KV heads of 128, 107.6, of which the bytes take 88.8.)
Q4Deal deal(const mlkv_q4cache *c, long long S, long long sum, long long warp_tiles, int nt_max, bool same)
{
    const int W = mlkv::q4_warps(c->d, c->G);
    const bool small = c->G <= 8;   // one accumulator
    // us: a launch's start and end; a tile per warp with one CTA and with two CTAs on the SM; records and merge
    // of warps, uneven ends included
    const float start = 3.f, one = small ? 1.05f : c->d == 64 ? 1.4f : 0.87f;
    const float two = small ? 1.75f : c->d == 64 ? 1.95f : 1.3f;
    const float warp_end = small ? 7.f : 10.f;
    const float sms = static_cast<float>(c->sm_count);
    const long long warps = static_cast<long long>(c->ctas_per_sm) * c->sm_count * W;
    const int whole = (nt_max + W - 1) / W;
    Q4Deal best = {whole, 1e30f};
    for (int k = 1, turns = whole;; k += (k + 7) / 8) {   // CTAs of the longest segment
        const int next = (whole + k - 1) / k;
        if (k > 1 && next == turns)
            continue;
        turns = next;
        const long long run = static_cast<long long>(turns) * W;
        const bool split = turns < whole;
        const long long pieces = (nt_max + run - 1) / run;
        // (uneven segments: their last runs are half full on average)
        const float ctas = same || !split ? static_cast<float>(S * pieces)
                                          : static_cast<float>(sum) / run + 0.5f * S;
        float t = start + merge_of(c, S, pieces).us;
        const int n = static_cast<int>(std::ceil(ctas / sms));   // CTAs on the busiest SM, two at a time
        if (same || n <= 2) {
            t += (n / 2) * turns * two + (n % 2) * turns * one + start * ((n + 1) / 2 - 1);
        } else {
            const float all = static_cast<float>(sum) / W + 0.5f * ctas;   // turns of all CTAs
            t += all * two / (2.f * sms) + 0.5f * turns * two + start * (ctas / (2.f * sms) - 1.f);
        }
        if (t < best.us)
            best = {turns, t};
        if (turns == 1)
            break;
    }
    const long long per_warp = warp_tiles / warps;
    const long long pieces = per_warp > 0 ? warp_pieces(nt_max, per_warp) : warps;
    const float t = start + warp_end + static_cast<float>(warp_tiles) / warps * two +
                    (pieces > mlkv::kQ4InlineMergePieces ? 1.5f : 0.f);
    if (per_warp > 0 && pieces <= mlkv::kCombineMaxPiecesHost && t < best.us)
        best = {0, t};
    return best;
}

}  // namespace

extern "C" {

int mlkv_q4_create(mlkv_q4cache_t *out, int n_layers, int n_q_heads, int head_dim,
                   const int *layer_owner, int kv_heads_per_owner, int batch, int max_seq)
{
    if (out == nullptr)
        return fail(MLKV_ERR_INVALID_ARG, "out is NULL");
    int rc = mlkv::validate_map(n_layers, n_q_heads, head_dim, layer_owner, kv_heads_per_owner, batch,
                                max_seq);
    if (rc != MLKV_OK)
        return rc;
    if (static_cast<long long>(batch) * kv_heads_per_owner > (1 << 24) || max_seq > (1 << 30))
        return fail(MLKV_ERR_UNSUPPORTED, "%d sequences of %d KV heads and %d positions exceed the "
                    "int32 indices", batch, kv_heads_per_owner, max_seq);
    mlkv_q4cache *c = new (std::nothrow) mlkv_q4cache();
    if (c == nullptr)
        return fail(MLKV_ERR_OOM, "out of host memory");
    c->l = n_layers;
    c->h = n_q_heads;
    c->d = head_dim;
    c->g = kv_heads_per_owner;
    c->G = n_q_heads / kv_heads_per_owner;
    c->b = batch;
    c->max_seq = max_seq;
    try {
        c->owner.assign(layer_owner, layer_owner + n_layers);
        c->slot.resize(n_layers);
    } catch (const std::bad_alloc &) {
        delete c;
        return fail(MLKV_ERR_OOM, "out of host memory");
    }
    for (int n = 0; n < n_layers; ++n)   // an owner comes before its readers
        c->slot[n] = c->owner[n] == n ? c->m++ : c->slot[c->owner[n]];
    c->row_bytes = mlkv::q4_row_bytes(max_seq, c->d);
    rc = mlkv::check_cache_bytes(static_cast<long long>(c->b) * c->g * c->m, c->row_bytes);
    if (rc != MLKV_OK) {
        delete c;
        return rc;
    }
    c->device = mlkv::current_device();
    DeviceGuard guard(c->device);
    cudaError_t e = cudaDeviceGetAttribute(&c->sm_count, cudaDevAttrMultiProcessorCount, c->device);
    if (e == cudaSuccess)
        e = mlkv::prepare_q4_decode(c->d, c->G, &c->ctas_per_sm);
    for (const bool windowed : {false, true})
        if (e == cudaSuccess)
            e = mlkv::prepare_prefill(c->d, windowed);
    if (e != cudaSuccess || c->ctas_per_sm < 1) {
        delete c;
        return e != cudaSuccess ? fail_cuda(e, "preparing the 4-bit cache's kernels")
                                : fail(MLKV_ERR_CUDA, "the 4-bit decode kernel cannot be resident");
    }
    const size_t rows = static_cast<size_t>(c->b) * c->g;
    c->cache_bytes = rows * c->m * c->row_bytes;
    // a record for each segment and each run of a launch
    const size_t records =
        rows + static_cast<size_t>(c->ctas_per_sm) * c->sm_count * mlkv::q4_warps(c->d, c->G);
    auto alloc = [&](void **ptr, size_t n) {
        if (e == cudaSuccess)
            e = cudaMalloc(ptr, n);
        if (e == cudaSuccess && ptr != reinterpret_cast<void **>(&c->part_o) &&
            ptr != reinterpret_cast<void **>(&c->part_lse))
            e = cudaMemset(*ptr, 0, n);
    };
    alloc(reinterpret_cast<void **>(&c->cache), c->cache_bytes);
    alloc(reinterpret_cast<void **>(&c->part_o), records * c->G * c->d * sizeof(float));
    alloc(reinterpret_cast<void **>(&c->part_lse), records * c->G * sizeof(float));
    alloc(reinterpret_cast<void **>(&c->counters), rows * sizeof(unsigned));
    alloc(reinterpret_cast<void **>(&c->err), sizeof(int));
    if (e == cudaSuccess)
        e = cudaDeviceSynchronize();
    if (e != cudaSuccess) {
        cudaGetLastError();
        const size_t need = c->cache_bytes;
        free_all(c);
        delete c;
        return fail(e == cudaErrorMemoryAllocation ? MLKV_ERR_OOM : MLKV_ERR_CUDA,
                    "allocating a %zu-byte 4-bit cache: %s", need, cudaGetErrorString(e));
    }
    *out = c;
    return MLKV_OK;
}

int mlkv_q4_destroy(mlkv_q4cache_t c)
{
    if (c == nullptr)
        return MLKV_OK;
    DeviceGuard guard(c->device);
    cudaDeviceSynchronize();
    free_all(c);
    delete c;
    return MLKV_OK;
}

int64_t mlkv_q4_bytes(mlkv_q4cache_t c)
{
    if (c == nullptr)
        return fail(MLKV_ERR_INVALID_ARG, "null cache handle");
    return static_cast<int64_t>(c->cache_bytes);
}

int mlkv_q4_append(mlkv_q4cache_t c, int layer, const void *K, const void *V, const int *seq_lens,
                   void *cuda_stream)
{
    int rc = check_layer(c, layer);
    if (rc != MLKV_OK)
        return rc;
    if (c->owner[layer] != layer)
        return MLKV_OK;   // Sec. 3: a layer without KV heads of its own stores nothing
    if (K == nullptr || V == nullptr || !aligned16(K) || !aligned16(V))
        return fail(MLKV_ERR_INVALID_ARG, "K and V must be non-NULL and 16-byte aligned");
    if ((rc = check_lens(c, seq_lens)) != MLKV_OK)
        return rc;
    DeviceGuard guard(c->device);
    return store(c, layer, K, V, 1, seq_lens, static_cast<cudaStream_t>(cuda_stream));
}

int mlkv_q4_load_prefix(mlkv_q4cache_t c, int layer, const void *K, const void *V, int len,
                        void *cuda_stream)
{
    int rc = check_layer(c, layer);
    if (rc != MLKV_OK)
        return rc;
    if (c->owner[layer] != layer)
        return MLKV_OK;
    if (len < 0 || len > c->max_seq)
        return fail(MLKV_ERR_RANGE, "prefix length %d outside [0, %d]", len, c->max_seq);
    if (len == 0)
        return MLKV_OK;
    DeviceGuard guard(c->device);
    if ((rc = check_prompt_kv(c, K, V)) != MLKV_OK)
        return rc;
    return store(c, layer, K, V, len, nullptr, static_cast<cudaStream_t>(cuda_stream));
}

int mlkv_q4_read(mlkv_q4cache_t c, int layer, void *K, void *V, int start, int len, void *cuda_stream)
{
    const int rc = check_layer(c, layer);
    if (rc != MLKV_OK)
        return rc;
    if (start < 0 || len < 0 || start > c->max_seq - len)
        return fail(MLKV_ERR_RANGE, "positions [%d, %d + %d) outside [0, %d)", start, start, len,
                    c->max_seq);
    if (len == 0)
        return MLKV_OK;
    if (K == nullptr || V == nullptr || !aligned16(K) || !aligned16(V))
        return fail(MLKV_ERR_INVALID_ARG, "K and V must be non-NULL and 16-byte aligned");
    const size_t bytes = static_cast<size_t>(c->b) * c->g * len * c->d * 2;
    if (overlap(K, bytes, V, bytes))
        return fail(MLKV_ERR_INVALID_ARG, "K and V overlap");
    DeviceGuard guard(c->device);
    mlkv::Q4ReadParams p;
    p.K = static_cast<__nv_bfloat16 *>(K);
    p.V = static_cast<__nv_bfloat16 *>(V);
    p.slot = slot_base(c, layer);
    p.row_bytes = c->row_bytes;
    p.b = c->b;
    p.g = c->g;
    p.start = start;
    p.len = len;
    const cudaError_t e = mlkv::launch_q4_read(c->d, p, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? MLKV_OK : fail_cuda(e, "4-bit read launch");
}

int mlkv_q4_decode_attention(mlkv_q4cache_t c, int layer, const void *Q, void *out,
                             const int *seq_lens, int window, int sinks, void *cuda_stream)
{
    int rc = check_layer(c, layer);
    if (rc != MLKV_OK)
        return rc;
    if (Q == nullptr || out == nullptr || !aligned16(Q) || !aligned16(out))
        return fail(MLKV_ERR_INVALID_ARG, "Q and out must be non-NULL and 16-byte aligned");
    const size_t qbytes = static_cast<size_t>(c->b) * c->h * c->d * 2;
    if (overlap(Q, qbytes, out, qbytes))
        return fail(MLKV_ERR_INVALID_ARG, "out overlaps Q");
    if ((rc = check_lens(c, seq_lens)) != MLKV_OK || (rc = mlkv::check_window(window, sinks)) != MLKV_OK)
        return rc;
    mlkv::clamp_window(c->max_seq, &window, &sinks);
    static thread_local mlkv::Q4DecodeParams p;
    static thread_local int real[MLKV_MAX_BATCH];   // a sequence's segments' tiles
    const int T = mlkv::q4_tile_tokens(c->d), W = mlkv::q4_warps(c->d, c->G);
    const long long S = static_cast<long long>(c->b) * c->g;
    const long long slots = static_cast<long long>(c->ctas_per_sm) * c->sm_count;   // resident CTAs
    int nt_min = 0x7fffffff, nt_max = 0;
    long long sum = 0;
    bool uniform = true;
    for (int beta = 0; beta < c->b; ++beta) {
        const int L = seq_lens[beta];
        const int nt = window > 0 ? mlkv::visible_tiles(L, window, sinks, T, mlkv::kQ4Block).nt
                                  : static_cast<int>((static_cast<unsigned>(L) + T - 1) / T);
        uniform = uniform && L == seq_lens[0];
        real[beta] = nt;
        p.seq_len[beta] = L;
        nt_min = std::min(nt_min, nt);
        nt_max = std::max(nt_max, nt);
        sum += nt;
    }
    p.uniform_len = uniform ? seq_lens[0] : 0;
    // The tiles are dealt out in equal runs.  A run a warp: tiles end to end, with three empty ones behind a
    // segment for the cost of its end (64 uneven sequences of up to 8192 positions, 8 KV heads of 128: 63.6,
    // 61.1, 60.1 us with 1, 2, 3, 59.7 to 61.2 with 4 to 8); every end is a record and its merge.  A run a
    // CTA: a segment's tiles filled up to whole runs, so that no run crosses a segment, of as many turns of
    // the warps as the estimate says; a whole segment needs no merge.  (Equal runs that cross segments
    // cost each CTA ~3 us an end: 16 uneven sequences of up to 1000, 8 KV heads of 128, 25.5 us, 9.0 now, 64
    // of them 39.2 and 18.5.)  Measured, us, a warp / a CTA: 32 sequences of 4096 37.9 / 33.2, 64 of 1000 24.1 /
    // 22.4, 20 of 4000 27.4 / 30.0, 64 uneven ones of up to 4000, 4 KV heads of 64, 18.7 / 17.2.
    const long long warp_tiles = c->g * (sum + static_cast<long long>(kEmpty) * c->b);
    int turns = deal(c, S, sum * c->g, warp_tiles, nt_max, nt_min == nt_max).turns;
    const bool warp_runs = turns == 0;
    int grid = static_cast<int>(slots);
    long long tiles = warp_tiles;
    long long pieces = 1;   // of a segment, at most
    p.empty_tiles = p.round_tiles = 0;
    if (warp_runs) {
        p.empty_tiles = kEmpty;
        pieces = warp_pieces(nt_max, warp_tiles / (slots * W));
    } else {
        // (as many runs as there are records for, and one merge takes; whole segments leave none)
        for (;; turns *= 2) {
            p.round_tiles = turns * W;
            tiles = 0;
            for (int beta = 0; beta < c->b; ++beta)
                tiles += (real[beta] + p.round_tiles - 1) / p.round_tiles;
            tiles *= c->g;
            pieces = (nt_max + p.round_tiles - 1) / p.round_tiles;
            if (pieces == 1 || (tiles <= slots * W && pieces <= mlkv::kCombineMaxPiecesHost))
                break;
        }
        grid = static_cast<int>(tiles);
        tiles *= p.round_tiles;
    }
    if (tiles > 0x7fffffffLL)
        return fail(MLKV_ERR_UNSUPPORTED, "%lld tiles exceed the int32 tile index", tiles);
    auto laid = [&](int beta) {   // tiles of one of beta's segments in the list
        return warp_runs ? real[beta] + kEmpty
                         : (real[beta] + p.round_tiles - 1) / p.round_tiles * p.round_tiles;
    };
    p.num_tiles = static_cast<int>(tiles);
    if (!uniform) {
        int at = 0;
        for (int beta = 0; beta < c->b; ++beta) {
            p.tile_start[beta] = at;
            at += c->g * laid(beta);
        }
        p.tile_start[c->b] = at;
    }
    p.deferred_merge = warp_runs ? pieces > mlkv::kQ4InlineMergePieces : merge_of(c, S, pieces).deferred;
    p.Q = static_cast<const __nv_bfloat16 *>(Q);
    p.out = static_cast<__nv_bfloat16 *>(out);
    p.slot = slot_base(c, layer);
    p.row_bytes = c->row_bytes;
    p.part_o = c->part_o;
    p.part_lse = c->part_lse;
    p.counters = c->counters;
    p.err = c->err;
    p.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(c->d)));
    p.b = c->b;
    p.h = c->h;
    p.g = c->g;
    p.G = c->G;
    p.window = window;
    p.sinks = sinks;
    DeviceGuard guard(c->device);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e = mlkv::launch_q4_decode(c->d, grid, warp_runs, p, stream);
    if (e != cudaSuccess)
        return fail_cuda(e, "4-bit decode launch");
    if (p.deferred_merge) {
        // The merge sees lengths whose plain tiling gives the launch's tiles.
        static thread_local mlkv::DecodeParams m;
        m.b = c->b;
        m.h = c->h;
        m.g = c->g;
        m.G = c->G;
        m.ml_layers = 0;
        m.num_tiles = p.num_tiles;
        m.uniform_len = uniform ? laid(0) * T : 0;
        if (!uniform)
            for (int beta = 0; beta < c->b; ++beta) {
                m.seq_len[beta] = laid(beta) * T;
                m.tile_start[beta] = p.tile_start[beta];
            }
        m.out = p.out;
        m.part_o = p.part_o;
        m.part_lse = p.part_lse;
        m.tile_tokens = T;
        m.decode_grid = grid * (warp_runs ? W : 1);
        // 256 threads a row take 4096 / d records a round trip to L2, 1024 four times as many but ~1 us
        // more for themselves: wide from the third round trip on (256 / 1024 threads, us: 171 records of
        // 12 heads of 64 12.9 / 11.4, 128 of 16 heads of 128 13.3 / 9.9; two: 38 of 16 heads of 128 9.9 / 9.6).
        const bool wide = pieces > 2 * 4096 / c->d;
        if ((e = mlkv::launch_combine(m, c->d, stream, true, wide)) != cudaSuccess)
            return fail_cuda(e, "combine launch");
    }
    return MLKV_OK;
}

int mlkv_q4_prefill(mlkv_q4cache_t c, int layer, const void *Q, const void *K, const void *V, void *out,
                    const int *prompt_lens, int s_max, int window, int sinks, void *cuda_stream)
{
    int rc = check_layer(c, layer);
    if (rc != MLKV_OK)
        return rc;
    if ((rc = mlkv::check_prefill_args(Q, out, prompt_lens, c->b, c->h, c->d, s_max, c->max_seq)) !=
            MLKV_OK ||
        (rc = mlkv::check_window(window, sinks)) != MLKV_OK)
        return rc;
    DeviceGuard guard(c->device);
    if ((rc = check_prompt_kv(c, K, V)) != MLKV_OK)
        return rc;
    const size_t qbytes = static_cast<size_t>(c->b) * s_max * c->h * c->d * 2;
    const size_t kvbytes = static_cast<size_t>(c->b) * c->g * s_max * c->d * 2;
    if (overlap(K, kvbytes, out, qbytes) || overlap(V, kvbytes, out, qbytes))
        return fail(MLKV_ERR_INVALID_ARG, "out overlaps K or V");
    mlkv::clamp_window(s_max, &window, &sinks);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    mlkv::PrefillCall a = {};
    a.Q = Q;
    a.K = K;
    a.V = V;
    a.out = out;
    a.prompt_lens = prompt_lens;
    a.err = c->err;
    a.b = c->b;
    a.h = c->h;
    a.g = c->g;
    a.d = c->d;
    a.s_max = s_max;
    a.sm_count = c->sm_count;
    a.direct = true;
    a.window = window;
    a.sinks = sinks;
    if ((rc = mlkv::issue_prefill(a, stream)) != MLKV_OK)
        return rc;
    return c->owner[layer] == layer ? store(c, layer, K, V, s_max, nullptr, stream) : MLKV_OK;
}

int mlkv_q4_sync_status(mlkv_q4cache_t c)
{
    if (c == nullptr)
        return fail(MLKV_ERR_INVALID_ARG, "null cache handle");
    DeviceGuard guard(c->device);
    cudaError_t e = cudaDeviceSynchronize();
    if (e != cudaSuccess)
        return fail_cuda(e, "cudaDeviceSynchronize");
    int word = 0;
    if ((e = cudaMemcpy(&word, c->err, sizeof(int), cudaMemcpyDeviceToHost)) != cudaSuccess)
        return fail_cuda(e, "reading the device error word");
    if (word != 0) {
        // A kernel stopped early: clear the word and the merge counters it may have left behind.
        cudaMemset(c->err, 0, sizeof(int));
        cudaMemset(c->counters, 0, static_cast<size_t>(c->b) * c->g * sizeof(unsigned));
        cudaDeviceSynchronize();
        return fail(MLKV_ERR_DEVICE, "a kernel reported device error bits 0x%x", word);
    }
    return MLKV_OK;
}

}  // extern "C"
