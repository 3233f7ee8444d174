// Host side of the operators for long caches: decode over a shared prefix, blocks' bounds, their selection and
// the decode over listed blocks, decode that adds up attention weights, eviction by them.  Argument checks,
// the split of the work, launches.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "mlkv_cache.h"
#include "mlkv_long.h"
#include "mlkv_plan.h"

using mlkv::aligned16;
using mlkv::check_layer;
using mlkv::check_seq_lens;
using mlkv::DeviceGuard;
using mlkv::driver_entry;
using mlkv::EncodeTiledFn;
using mlkv::fail;
using mlkv::fail_cuda;
using mlkv::overlap;

namespace {

// Bits of mlkv_cache::long_ready.
enum : unsigned { kReadyPieces = 1, kReadySelect = 32, kReadyEvict = 64, kReadyShared = 128 };   // pieces: 5 bits

bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

size_t query_bytes(const mlkv_cache *c) { return static_cast<size_t>(c->b) * c->h * c->d * 2; }

int check_queries(const mlkv_cache *c, const void *Q, const void *out)
{
    if (Q == nullptr || out == nullptr || !aligned16(Q) || !aligned16(out))
        return fail(MLKV_ERR_INVALID_ARG, "Q and out must be non-NULL and 16-byte aligned");
    if (overlap(Q, query_bytes(c), out, query_bytes(c)))
        return fail(MLKV_ERR_INVALID_ARG, "out overlaps Q");
    return MLKV_OK;
}

const CUtensorMap *rows64(const mlkv_cache *c) { return &c->variants.front().tmap_rows; }

int prepare_pieces(mlkv_cache *c, int mode)
{
    const unsigned bit = kReadyPieces << mode;
    if (c->long_ready & bit)
        return MLKV_OK;
    const cudaError_t e = mlkv::prepare_pieces(c->d, c->G, mode, &c->piece_ctas);
    if (e != cudaSuccess)
        return fail_cuda(e, "preparing the piece kernel");
    if (c->piece_ctas < 1)
        return fail(MLKV_ERR_CUDA, "the piece kernel cannot be resident");
    c->long_ready |= bit;
    return MLKV_OK;
}

// How the segments, nt(beta) tiles each, are cut into pieces: the least estimated time, in us.  A
// launch takes 4.5, and what is longer of its bytes at the rate of HBM and its longest piece; pieces beyond one wave
// of resident CTAs half a piece more where segments are split (whole ones end evenly enough).  Split segments
// are merged by the CTA that ends last, a round trip to L2 for every 8 records, or by a launch of their own.  Never more
// pieces than there are records.  pre: records that every merge has besides; hbm_tiles: tiles that come from HBM, the
// others from L2 (14 TB/s, groups above 8 heads 10); -1: all.
struct Cut {
    bool defer;
    int records;   // of a segment, at most
    int tiles;     // of a piece
    double us;     // estimated
};
struct CutRules {
    int n;                   // query rows
    long long most_pieces;   // records that there is room for
    bool always_apart;       // a merge of its own in any case
    bool never_here;         // no merge by the CTA that ends last
    int pre;
    double hbm_tiles;
};
template <typename Tiles>
Cut plan_cut(const mlkv_cache *c, const CutRules &r, const Tiles &nt)
{
    long long total = 0;
    int longest = 1, shortest = 0x7fffffff;
    for (int beta = 0; beta < r.n; ++beta) {
        const int n = nt(beta);
        total += n;
        longest = std::max(longest, n);
        shortest = std::min(shortest, n);
    }
    total *= c->g;
    const long long slots = static_cast<long long>(c->piece_ctas) * c->sm_count;
    const int stages = mlkv::piece_stages(c->d);
    // us: a tile of a CTA alone on its SM; all tiles at the rate of HBM; a record's part of an inline merge
    const double tile = c->d == 64 ? 0.33 : c->G <= 8 ? 0.45 : 0.72;
    const double from_hbm = r.hbm_tiles < 0 ? total : r.hbm_tiles;
    const double bytes = std::max(from_hbm / 6.7e6, total / (c->G <= 8 ? 14e6 : 10e6)) * 256.0 * c->d;
    const double record = 0.1 * c->G * c->d / 512;
    const int inline_most = mlkv::piece_max_records(c->d, c->G) - r.pre;
    Cut best = {r.always_apart, 1, longest, 1e30};
    for (int want = 1, tiles = longest;; want += (want + 3) / 4) {   // pieces of the longest segment
        const int next = (longest + want - 1) / want;
        if (want > 1 && next == tiles)
            continue;
        tiles = next;
        long long n = 0;
        if (shortest == longest)
            n = static_cast<long long>(r.n) * ((longest + tiles - 1) / tiles);
        else
            for (int beta = 0; beta < r.n; ++beta)
                n += (nt(beta) + tiles - 1) / tiles;
        n *= c->g;
        const int pieces = (longest + tiles - 1) / tiles, records = pieces + r.pre;
        if (want > 1 && (n > std::min(r.most_pieces, 4 * slots) || records > mlkv::kDeferMaxRecords))
            break;
        const double rounds = (tiles + stages - 1) / stages;   // (a short piece's tiles come at once)
        double t = 4.5 + std::max(bytes, 1.15 * std::max(tiles * tile, rounds * 1.2));
        if (n > slots && pieces > 1)
            t += 0.5 * tiles * tile + 2.0;
        const double here = records <= 1 ? 0.0 : 2.5 + record * records, apart = 4.5;
        const bool defer = r.always_apart ||
                           (records > 1 && (r.never_here || here > apart || records > inline_most));
        t += defer ? apart : here;
        if (t < best.us)
            best = {defer, records, tiles, t};
        if (best.us <= 4.5 + bytes + 2.5)   // no split takes less
            break;
        if (tiles == 1)
            break;
    }
    return best;
}

// Lays the pieces of a plan out: p.tiles and p.first.
template <typename Tiles>
void lay_pieces(const mlkv_cache *c, mlkv::PieceParams &p, const Cut &split, const Tiles &nt)
{
    p.tiles = split.tiles;
    // Uneven rows the longest first, to one part in 255: what starts last is short (48 sequences of up to 3000
    // positions, 8 KV heads of 128, 56.4 us as they come, 53.1 so; 100 of up to 4000 132.4, 123.1).
    int longest = 0, shortest = 0x7fffffff, count[257] = {};
    for (int i = 0; i < p.n; ++i) {
        longest = std::max(longest, nt(i));
        shortest = std::min(shortest, nt(i));
    }
    p.ordered = longest > shortest ? 1 : 0;
    if (p.ordered) {
        const int step = longest / 255 + 1;
        for (int i = 0; i < p.n; ++i)
            ++count[256 - nt(i) / step];
        for (int k = 1; k < 257; ++k)
            count[k] += count[k - 1];
        for (int i = 0; i < p.n; ++i)   // (256 - nt / step is at least 1)
            p.order[count[255 - nt(i) / step]++] = static_cast<uint16_t>(i);
    }
    long long at = 0;
    for (int i = 0; i < p.n; ++i) {
        p.first[i] = static_cast<int>(at);
        at += static_cast<long long>(c->g) * ((nt(p.ordered ? p.order[i] : i) + p.tiles - 1) / p.tiles);
    }
    p.first[p.n] = static_cast<int>(at);
}

void fill_pieces(const mlkv_cache *c, int layer, const void *Q, void *out, const int *seq_lens,
                 mlkv::PieceParams &p)
{
    p.Q = static_cast<const __nv_bfloat16 *>(Q);
    p.out = static_cast<__nv_bfloat16 *>(out);
    p.part_o = c->part_o;
    p.part_lse = c->part_lse;
    p.counters = c->counters;
    p.err = c->err;
    p.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(c->d)));
    p.b = p.n = c->b;
    p.scattered = 0;
    p.h = c->h;
    p.g = c->g;
    p.G = c->G;
    p.slot = c->slot[layer];
    p.pre_o = p.pre_lse = nullptr;
    p.pre_chunks = p.early = p.defer = 0;
    p.blocks = nullptr;
    p.n_blocks = 0;
    p.scores = nullptr;
    p.score_stride = 0;
    std::memcpy(p.seq_len, seq_lens, sizeof(int) * c->b);
}

// A stream under capture takes no allocation: scratch that would have to grow is refused there.
int scratch(mlkv_cache *c, size_t floats, const char *what, cudaStream_t stream)
{
    if (floats <= c->fused_part_floats)
        return MLKV_OK;
    cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(stream, &st) != cudaSuccess || st != cudaStreamCaptureStatusNone) {
        cudaGetLastError();
        return fail(MLKV_ERR_UNSUPPORTED, "%s: %zu bytes to allocate while the stream is captured; make this "
                    "call once outside", what, floats * sizeof(float));
    }
    return mlkv::grow_scratch(c, floats, what);
}

// The piece launch, and the merge's where it is one of its own.
int decode_pieces(const mlkv_cache *c, int mode, mlkv::PieceParams &p, const Cut &split,
                  const CUtensorMap *tmap_prefix, cudaStream_t stream)
{
    p.defer = split.defer ? 1 : 0;
    cudaError_t e = mlkv::launch_pieces(c->d, mode, rows64(c), tmap_prefix, p, stream);
    if (e != cudaSuccess)
        return fail_cuda(e, "decode launch");
    if (p.defer && (e = mlkv::launch_merge_pieces(c->d, mode, p, split.records, stream)) != cudaSuccess)
        return fail_cuda(e, "merge launch");
    return MLKV_OK;
}

// Scattered rows' records, behind `before` floats of the scratch (rounded up to 16 bytes).
int own_records(mlkv_cache *c, mlkv::PieceParams &p, size_t before, cudaStream_t stream)
{
    before = (before + 3) / 4 * 4;
    const size_t rows = static_cast<size_t>(p.first[p.n]) * c->G;
    const int rc = scratch(c, before + rows * (c->d + 1), "records of a prompt's tokens", stream);
    if (rc != MLKV_OK)
        return rc;
    p.part_o = c->fused_part + before;
    p.part_lse = p.part_o + rows * c->d;
    return MLKV_OK;
}

}  // namespace

int mlkv::check_same_model(const mlkv_cache *c, const mlkv_cache *other, const char *what)
{
    if (other == nullptr)
        return fail(MLKV_ERR_INVALID_ARG, "null %s handle", what);
    if (other->l != c->l || other->h != c->h || other->d != c->d || other->g != c->g ||
        other->owner != c->owner)
        return fail(MLKV_ERR_MAP, "the %s has other layers or heads", what);
    if (other->device != c->device)
        return fail(MLKV_ERR_INVALID_ARG, "the %s lies on another device", what);
    return MLKV_OK;
}

int mlkv::check_prefix(const mlkv_cache *c, const mlkv_cache *prefix, const int *prefix_of,
                       const int *prefix_lens)
{
    const int rc = check_same_model(c, prefix, "prefix cache");
    if (rc != MLKV_OK)
        return rc;
    if (prefix_of == nullptr || prefix_lens == nullptr)
        return fail(MLKV_ERR_INVALID_ARG, "prefix_of and prefix_lens must be non-NULL");
    for (int beta = 0; beta < c->b; ++beta)
        if (prefix_of[beta] < -1 || prefix_of[beta] >= prefix->b)
            return fail(MLKV_ERR_RANGE, "prefix_of[%d] = %d outside [-1, %d)", beta, prefix_of[beta], prefix->b);
    for (int x = 0; x < prefix->b; ++x)
        if (prefix_lens[x] < 0 || prefix_lens[x] > prefix->max_seq)
            return fail(MLKV_ERR_RANGE, "prefix_lens[%d] = %d outside [0, %d]", x, prefix_lens[x],
                        prefix->max_seq);
    return MLKV_OK;
}

int mlkv::decode_rows(mlkv_cache *c, int layer, const mlkv_cache *prefix, const int *prefix_lens,
                      const PrefixRows &rows, const void *Q, void *out, cudaStream_t stream, PromptStep *step)
{
    int rc = ::prepare_pieces(c, mlkv::kPieceSuffix);
    if (rc != MLKV_OK)
        return rc;
    static thread_local mlkv::PieceParams p;
    static thread_local mlkv::SharedPrefillParams u;
    static thread_local bool read[MLKV_MAX_BATCH];
    fill_pieces(c, layer, Q, out, rows.len, p);   // (scattered rows are no fewer than sequences)
    p.n = rows.n;
    p.scattered = rows.scattered;
    if (rows.scattered) {
        std::memcpy(p.seq_len, rows.len, sizeof(int) * rows.n);
        std::memcpy(p.q_row, rows.q_row, sizeof(uint16_t) * rows.n);
        std::memcpy(p.seq, rows.seq, sizeof(uint16_t) * rows.n);
    }
    // Each sequence's prefix and positions end to end, if that is no longer than the prefixes apart: few sequences a
    // prefix.
    double hbm = 0, bytes = 0;   // tiles of 64 positions that are read once; bytes of the suffixes
    for (int x = 0; x < prefix->b; ++x)
        read[x] = false;
    for (int beta = 0; beta < rows.n; ++beta) {
        const int x = rows.prefix[beta];
        p.pre_len[beta] = x >= 0 ? prefix_lens[x] : 0;
        p.pre_place[beta] = static_cast<uint16_t>(x >= 0 ? x : 0);
        hbm += (rows.len[beta] + 63) / 64;
        bytes += 4.0 * c->g * c->d * rows.len[beta];
        if (x >= 0 && !read[x]) {
            read[x] = true;
            hbm += (prefix_lens[x] + 63) / 64;
        }
    }
    const auto joined = [&](int beta) { return mlkv::piece_tiles<mlkv::kPieceJoined>(p, beta); };
    // (scattered rows have no counters, and their records in the scratch)
    const long long room = rows.scattered ? 0x7fffffff : c->records;
    const Cut end_to_end = plan_cut(c, {rows.n, room, false, rows.scattered != 0, 0, hbm * c->g}, joined);
    // Places: the sequences of prefix 0, then those of prefix 1, ...  Where every prefix's sequences are
    // neighbours already, a sequence's place is its own number.
    const int L1 = 128 / c->G, np = prefix->b;
    static thread_local int n_kt[MLKV_MAX_BATCH], pairs[MLKV_MAX_BATCH];
    static thread_local mlkv::PrefixPlan plan;
    std::fill(u.group_n, u.group_n + np, static_cast<uint16_t>(0));
    auto of = [&](int beta) {
        return rows.prefix[beta] >= 0 && prefix_lens[rows.prefix[beta]] > 0 ? rows.prefix[beta] : -1;
    };
    bool neighbours = rows.scattered == 0;
    int places = 0;
    for (int beta = 0; beta < rows.n; ++beta) {
        const int x = of(beta);
        if (x < 0)
            continue;
        ++places;
        if (u.group_n[x]++ == 0)
            u.group_at[x] = static_cast<uint16_t>(beta);
        else
            neighbours = neighbours && of(beta - 1) == x;
    }
    u.scattered = neighbours ? 0 : 1;
    int most_kt = 0;
    for (int x = 0; x < np; ++x) {
        n_kt[x] = u.group_n[x] > 0 ? (prefix_lens[x] + 127) / 128 : 0;
        pairs[x] = (u.group_n[x] + 2 * L1 - 1) / (2 * L1) * c->g;
        most_kt = std::max(most_kt, n_kt[x]);
    }
    if (most_kt > 0)
        plan = mlkv::plan_prefix(n_kt, pairs, np, c->sm_count, c->d, bytes, mlkv::kFusedMaxChunks);
    // The prefixes for as many sequences at a time as have 16 heads together, beside the suffixes in their launch: read
    // from L2 again for every group of them, and merged by a launch.  us: 9, and what is longest of the bytes from HBM,
    // those through the SMs (8.5 TB/s) and a unit; half the longest suffix more where those are uneven.  Measured, us, end
    // to end / by groups / by the prefix kernel: 4 sequences behind 16000 positions, 8 KV heads of 128, 26 / 21 / 27,
    // 8 of them 37 / 26 / 32, 16 of them 64 / 37 / 34; 16 behind 4000, 12 KV heads of 64, 32 / 11 / 15.  (What is taken
    // goes by the estimates: of 26 shapes it is within 3% of the best form in 22, and 8 to 29% behind in four.)
    const int S1 = 16 / c->G;
    double grouped_us = 1e30;
    int unit_tiles = 8;
    if (most_kt > 0 && !rows.scattered) {
        double from_l2 = 0, in_units = 0;
        int longest = 1, shortest = 0x7fffffff;
        for (int beta = 0; beta < rows.n; ++beta) {
            const int nt = (rows.len[beta] + 63) / 64;
            from_l2 += nt;
            longest = std::max(longest, nt);
            shortest = std::min(shortest, nt);
        }
        for (int x = 0; x < np; ++x)
            if (u.group_n[x] > 0)
                in_units += static_cast<double>((prefix_lens[x] + 63) / 64) * ((u.group_n[x] + S1 - 1) / S1);
        from_l2 += in_units;
        // as many units as CTAs are resident, at most; no more than 255 chunks of a prefix
        unit_tiles = std::max({unit_tiles, static_cast<int>(in_units * c->g / (1.75 * c->sm_count)) + 1,
                               (2 * most_kt + 254) / 255});
        long long units = 0;
        for (int x = 0; x < np; ++x)
            if (u.group_n[x] > 0)
                units += static_cast<long long>(((prefix_lens[x] + 63) / 64 + unit_tiles - 1) / unit_tiles) *
                         ((u.group_n[x] + S1 - 1) / S1) * c->g;
        const double tile_bytes = 256.0 * c->d * c->g, tile = c->d == 64 ? 0.34 : 0.72;
        if (units <= mlkv::kPieceMaxUnits)
            grouped_us = 9 + std::max({hbm / 6.3e6 * tile_bytes, from_l2 / 8.5e6 * tile_bytes,
                                       1.15 * unit_tiles * tile}) +
                         (longest > shortest + unit_tiles ? 0.5 * longest * tile : 0.0);
    }
    const double apart_us = most_kt > 0 ? plan.us : 1e30;
    const bool grouped = grouped_us < std::min(apart_us, end_to_end.us);
    if (step != nullptr && std::min(apart_us, end_to_end.us) >= step->most_us)   // (scattered: no groups)
        return MLKV_OK;
    // Scratch that cannot be had: a prompt goes on without its rows.
    const auto no_scratch = [&](int err) {
        return step != nullptr && (err == MLKV_ERR_UNSUPPORTED || err == MLKV_ERR_OOM) ? MLKV_OK : err;
    };
    const auto begin = [&]() {
        if (step == nullptr)
            return MLKV_OK;
        step->issued = true;
        return step->store != nullptr ? step->store(*step, stream) : MLKV_OK;
    };
    if (!grouped && end_to_end.us <= apart_us) {
        if ((rc = ::prepare_pieces(c, mlkv::kPieceJoined)) != MLKV_OK)
            return rc;
        p.prefix_b = prefix->b;
        lay_pieces(c, p, end_to_end, joined);
        if (rows.scattered && (rc = own_records(c, p, 0, stream)) != MLKV_OK)
            return no_scratch(rc);
        if ((rc = begin()) != MLKV_OK)
            return rc;
        c->last_prefix_form = mlkv::kFormJoined;
        c->last_prefix_launches = end_to_end.defer ? 2 : 1;
        return decode_pieces(c, mlkv::kPieceJoined, p, end_to_end, rows64(prefix), stream);
    }
    if (neighbours) {
        for (int beta = 0; beta < rows.n; ++beta)
            p.pre_place[beta] = static_cast<uint16_t>(beta);
        places = rows.n;
    } else {
        int at = 0;
        for (int x = 0; x < np; ++x) {
            u.group_at[x] = static_cast<uint16_t>(at);
            at += u.group_n[x];
            u.group_n[x] = 0;
        }
        for (int beta = 0; beta < rows.n; ++beta)
            if (of(beta) >= 0) {
                const int place = u.group_at[of(beta)] + u.group_n[of(beta)]++;
                p.pre_place[beta] = static_cast<uint16_t>(place);
                u.seq[place] = rows.scattered ? rows.q_row[beta] : static_cast<uint16_t>(beta);
            }
    }
    if (!grouped && !(c->long_ready & kReadyShared)) {
        const cudaError_t e = mlkv::prepare_shared(c->d, true);
        if (e != cudaSuccess)
            return fail_cuda(e, "preparing the decode over a shared prefix");
        c->long_ready |= kReadyShared;
    }
    // chunks of a prefix, in key tiles of 128 positions, or of 64 by groups
    const int kc = grouped ? unit_tiles : plan.kc;
    const auto chunks = [&](int x) {
        return ((grouped ? (prefix_lens[x] + 63) / 64 : (prefix_lens[x] + 127) / 128) + kc - 1) / kc;
    };
    int cmax = 0;
    for (int x = 0; x < np; ++x)
        if (n_kt[x] > 0)
            cmax = std::max(cmax, chunks(x));
    const size_t records = static_cast<size_t>(places) * c->g * cmax * c->G;
    for (int beta = 0; beta < rows.n; ++beta) {
        const int x = of(beta);
        p.pre_n[beta] = static_cast<uint16_t>(x < 0 ? 0 : chunks(x));
    }
    const auto own = [&](int beta) { return mlkv::piece_tiles<mlkv::kPieceSuffix>(p, beta); };
    const Cut split = plan_cut(c, {rows.n, room, grouped || plan.beside, rows.scattered != 0, cmax, -1}, own);
    lay_pieces(c, p, split, own);
    if ((rc = rows.scattered ? own_records(c, p, records * (c->d + 1), stream)
                             : scratch(c, records * (c->d + 1), "records of the shared prefix", stream)) != MLKV_OK)
        return no_scratch(rc);
    u.part = c->fused_part;
    u.part_lse = u.part + records * c->d;
    p.pre_o = u.part;
    p.pre_lse = u.part_lse;
    p.pre_chunks = cmax;
    if (grouped) {
        if ((rc = ::prepare_pieces(c, mlkv::kPieceGroups)) != MLKV_OK)
            return rc;
        std::memcpy(p.prefix_len, prefix_lens, sizeof(int) * np);
        for (int beta = 0; beta < rows.n; ++beta)
            if (of(beta) >= 0)
                p.place_row[p.pre_place[beta]] = static_cast<uint16_t>(beta);
        p.prefix_b = np;
        p.unit_tiles = kc;
        p.n_units = 0;
        for (int x = 0; x < np; ++x)
            for (int j = 0; j < c->g && n_kt[x] > 0; ++j)
                for (int ch = 0; ch < chunks(x); ++ch)
                    for (int s = 0; s < u.group_n[x]; s += S1) {   // neighbours read the same tiles
                        p.units[p.n_units] = static_cast<uint32_t>(x) | (static_cast<uint32_t>(ch) << 10) |
                                             (static_cast<uint32_t>(j) << 18) |
                                             (static_cast<uint32_t>(std::min(S1, u.group_n[x] - s) - 1) << 26);
                        p.unit_place[p.n_units++] = static_cast<uint16_t>(u.group_at[x] + s);
                    }
        c->last_prefix_form = mlkv::kFormGroups;
        c->last_prefix_launches = 2;
        return decode_pieces(c, mlkv::kPieceGroups, p, split, rows64(prefix), stream);
    }
    p.early = 1;
    // The queries [b][h][D] as (channel, head in group, group, 1, sequence): a box of 64 channels x G heads x
    // min(L1, b) neighbours is a tile's rows, one of 64 channels x G heads a scattered sequence's.
    static EncodeTiledFn encode = driver_entry<EncodeTiledFn>("cuTensorMapEncodeTiled");
    if (encode == nullptr)
        return fail(MLKV_ERR_CUDA, "cuTensorMapEncodeTiled is unavailable from the driver");
    CUtensorMap tmap_q;
    const cuuint64_t row = static_cast<cuuint64_t>(c->h) * c->d * 2;
    const cuuint64_t dims[5] = {static_cast<cuuint64_t>(c->d), static_cast<cuuint64_t>(c->G),
                                static_cast<cuuint64_t>(c->g), 1u, static_cast<cuuint64_t>(rows.q_rows)};
    const cuuint64_t strides[4] = {static_cast<cuuint64_t>(c->d) * 2,
                                   static_cast<cuuint64_t>(c->G) * c->d * 2, row, row};
    const cuuint32_t box[5] = {64u, static_cast<cuuint32_t>(c->G), 1u, 1u,
                               static_cast<cuuint32_t>(neighbours ? std::min(L1, rows.n) : 1)};
    const cuuint32_t estr[5] = {1u, 1u, 1u, 1u, 1u};
    const CUresult r = encode(&tmap_q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void *>(Q), dims,
                              strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS)
        return fail(MLKV_ERR_CUDA, "cuTensorMapEncodeTiled(Q) failed (CUresult %d)",
                    static_cast<int>(r));
    const CUtensorMap *tmap_kv = nullptr;
    for (auto &v : prefix->variants)
        if (v.v->tile_tokens == 128)
            tmap_kv = &v.tmap;
    if (tmap_kv == nullptr)
        return fail(MLKV_ERR_UNSUPPORTED, "no 128-position cache map for d=%d", c->d);
    u.tmap_p = *tmap_kv;
    u.out = nullptr;
    u.err = c->err;
    u.scale_log2 = p.scale_log2;
    u.b = c->b;
    u.h = c->h;
    u.g = c->g;
    u.G = c->G;
    u.s_max = prefix->max_seq;
    u.slot = p.slot;
    u.head_pairs = 0;
    u.sm_count = plan.sms;
    u.window = u.sinks = 0;
    u.kv_direct = 0;
    u.fused_L = rows.n;
    u.fused_L1 = L1;
    u.fused_nblk = 1;
    u.fused_kc = kc;
    u.fused_cmax = cmax;
    u.fused_early = 0;
    u.fused_combine_w = 1;
    u.q_host = nullptr;
    u.prefix_b = np;
    std::memcpy(u.prompt_len, prefix_lens, sizeof(int) * np);
    if ((rc = begin()) != MLKV_OK)
        return rc;
    c->last_prefix_form = plan.beside ? mlkv::kFormBeside : mlkv::kFormKernel;
    c->last_prefix_launches = split.defer ? 2 : 1;
    int n = 0;
    auto issue = [&]() {
        u.n_units = n;
        n = 0;
        ++c->last_prefix_launches;
        return mlkv::launch_shared(c->d, true, &tmap_q, tmap_kv, tmap_kv, u, stream);
    };
    for (int x = 0; x < np; ++x) {
        const int nblk = (u.group_n[x] + 2 * L1 - 1) / (2 * L1);
        for (int j = 0; j < c->g && n_kt[x] > 0; ++j)
            for (int ch = 0; ch * kc < n_kt[x]; ++ch)
                for (int blk = 0; blk < nblk; ++blk) {   // neighbours read the same tiles
                    u.units[n] = static_cast<uint32_t>(x) | (static_cast<uint32_t>(ch) << 10) |
                                 (static_cast<uint32_t>(blk) << 18) | (static_cast<uint32_t>(j) << 24);
                    if (++n == mlkv::kPrefixMaxUnits) {
                        const cudaError_t e = issue();
                        if (e != cudaSuccess)
                            return fail_cuda(e, "shared prefix launch");
                    }
                }
    }
    if (n > 0) {
        const cudaError_t e = issue();
        if (e != cudaSuccess)
            return fail_cuda(e, "shared prefix launch");
    }
    return decode_pieces(c, mlkv::kPieceSuffix, p, split, rows64(c), stream);
}

extern "C" {

int mlkv_decode_attention_prefix(mlkv_cache_t c, int layer, mlkv_cache_t prefix, const int *prefix_of,
                                 const int *prefix_lens, const void *Q, void *out, const int *seq_lens,
                                 void *cuda_stream)
{
    int rc = check_layer(c, layer);
    if (rc != MLKV_OK || (rc = mlkv::check_prefix(c, prefix, prefix_of, prefix_lens)) != MLKV_OK ||
        (rc = check_queries(c, Q, out)) != MLKV_OK || (rc = check_seq_lens(c, seq_lens)) != MLKV_OK)
        return rc;
    if (c->g > 255)
        return fail(MLKV_ERR_UNSUPPORTED, "the decode over a shared prefix handles at most 255 KV heads");
    static thread_local mlkv::PrefixRows rows;
    rows.n = rows.q_rows = c->b;
    rows.scattered = 0;
    std::memcpy(rows.len, seq_lens, sizeof(int) * c->b);
    std::memcpy(rows.prefix, prefix_of, sizeof(int) * c->b);
    DeviceGuard guard(c->device);
    return mlkv::decode_rows(c, layer, prefix, prefix_lens, rows, Q, out,
                             static_cast<cudaStream_t>(cuda_stream));
}

int mlkv_block_bounds(mlkv_cache_t c, int layer, const int *first, const int *seq_lens, void *bounds,
                      float *scales, void *cuda_stream)
{
    int rc = check_layer(c, layer);
    if (rc != MLKV_OK)
        return rc;
    if (c->owner[layer] != layer)
        return MLKV_OK;   // its owner's bounds are these
    if ((rc = check_seq_lens(c, seq_lens)) != MLKV_OK)
        return rc;
    if (bounds == nullptr || scales == nullptr || !aligned16(bounds) || !aligned4(scales))
        return fail(MLKV_ERR_INVALID_ARG, "bounds must be 16-byte and scales 4-byte aligned, neither NULL");
    static thread_local mlkv::BoundsParams p;
    p.n_blocks = static_cast<int>((static_cast<unsigned>(c->max_seq) + 63) / 64);
    const size_t blocks = static_cast<size_t>(c->b) * c->g * p.n_blocks;
    if (overlap(bounds, blocks * 2 * c->d, scales, blocks * 4))
        return fail(MLKV_ERR_INVALID_ARG, "bounds overlap scales");
    long long ctas = 0, total = 0;
    for (int beta = 0; beta < c->b; ++beta) {
        const int f = first != nullptr ? first[beta] : 0;
        if (f < 0 || f > seq_lens[beta])
            return fail(MLKV_ERR_RANGE, "first[%d] = %d outside [0, %d]", beta, f, seq_lens[beta]);
        p.seq_len[beta] = seq_lens[beta];
        p.first[beta] = f;
        total += static_cast<long long>(c->g) * ((seq_lens[beta] + 63) / 64 - f / 64);
    }
    p.per_cta = mlkv::bounds_per_cta(total, c->sm_count);
    for (int beta = 0; beta < c->b; ++beta) {
        p.start[beta] = static_cast<int>(std::min(ctas, 0x7fffffffLL));
        ctas += static_cast<long long>(c->g) *
                (((seq_lens[beta] + 63) / 64 - p.first[beta] / 64 + p.per_cta - 1) / p.per_cta);
    }
    if (ctas == 0)
        return MLKV_OK;
    if (ctas > 0x7fffffffLL)
        return fail(MLKV_ERR_UNSUPPORTED, "%lld CTAs exceed a launch", ctas);
    p.start[c->b] = static_cast<int>(ctas);
    const size_t slot = c->cache_bytes / c->m;
    p.K = reinterpret_cast<const __nv_bfloat16 *>(static_cast<char *>(c->cache) + slot * c->slot[layer]);
    p.bounds = static_cast<int8_t *>(bounds);
    p.scales = scales;
    p.b = c->b;
    p.g = c->g;
    p.max_seq = c->max_seq;
    DeviceGuard guard(c->device);
    const cudaError_t e = mlkv::launch_bounds(c->d, p, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? MLKV_OK : fail_cuda(e, "block bounds launch");
}

int mlkv_select_blocks(mlkv_cache_t c, int layer, const void *Q, const void *bounds, const float *scales,
                       const int *seq_lens, int n_select, int n_first, int n_last, int *blocks,
                       void *cuda_stream)
{
    int rc = check_layer(c, layer);
    if (rc != MLKV_OK)
        return rc;
    if (Q == nullptr || !aligned16(Q) || bounds == nullptr || !aligned16(bounds) || scales == nullptr ||
        !aligned4(scales) || blocks == nullptr || !aligned4(blocks))
        return fail(MLKV_ERR_INVALID_ARG, "Q and bounds must be 16-byte, scales and blocks 4-byte aligned, none NULL");
    if ((rc = check_seq_lens(c, seq_lens)) != MLKV_OK)
        return rc;
    if (n_select < 1 || n_first < 0 || n_last < 0 || n_first > n_select - n_last)
        return fail(MLKV_ERR_INVALID_ARG, "%d blocks cannot hold the %d first and the %d last ones", n_select,
                    n_first, n_last);
    static thread_local mlkv::SelectParams p;
    p.n_blocks = static_cast<int>((static_cast<unsigned>(c->max_seq) + 63) / 64);
    const size_t n = static_cast<size_t>(c->b) * c->g, out_bytes = n * n_select * 4;
    if (overlap(blocks, out_bytes, Q, query_bytes(c)) ||
        overlap(blocks, out_bytes, bounds, n * p.n_blocks * 2 * c->d) ||
        overlap(blocks, out_bytes, scales, n * p.n_blocks * 4))
        return fail(MLKV_ERR_INVALID_ARG, "blocks overlap an input");
    int most = 0;
    for (int beta = 0; beta < c->b; ++beta) {
        p.seq_len[beta] = seq_lens[beta];
        most = std::max(most, static_cast<int>((static_cast<unsigned>(seq_lens[beta]) + 63) / 64));
    }
    if (most > mlkv::select_max_blocks())
        return fail(MLKV_ERR_UNSUPPORTED, "%d blocks of a sequence: a selection handles %d", most,
                    mlkv::select_max_blocks());
    if (n > (1u << 24))
        return fail(MLKV_ERR_UNSUPPORTED, "%zu KV heads exceed a launch", n);
    p.Q = static_cast<const __nv_bfloat16 *>(Q);
    p.bounds = static_cast<const int8_t *>(bounds);
    p.scales = scales;
    p.blocks = blocks;
    p.b = c->b;
    p.h = c->h;
    p.g = c->g;
    p.G = c->G;
    p.n_select = n_select;
    p.n_first = n_first;
    p.n_last = n_last;
    DeviceGuard guard(c->device);
    cudaError_t e = cudaSuccess;
    if (!(c->long_ready & kReadySelect) && (e = mlkv::prepare_select(c->d)) == cudaSuccess)
        c->long_ready |= kReadySelect;
    if (e == cudaSuccess)
        e = mlkv::launch_select(c->d, p, most, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? MLKV_OK : fail_cuda(e, "block selection launch");
}

int mlkv_decode_attention_blocks(mlkv_cache_t c, int layer, const void *Q, void *out, const int *seq_lens,
                                 const int *blocks, int n_blocks, void *cuda_stream)
{
    int rc = check_layer(c, layer);
    if (rc != MLKV_OK || (rc = check_queries(c, Q, out)) != MLKV_OK ||
        (rc = check_seq_lens(c, seq_lens)) != MLKV_OK)
        return rc;
    if (blocks == nullptr || !aligned4(blocks) || n_blocks < 1)
        return fail(MLKV_ERR_INVALID_ARG, "blocks must be non-NULL and 4-byte aligned, at least one");
    const size_t segments = static_cast<size_t>(c->b) * c->g;
    if (overlap(blocks, segments * n_blocks * 4, out, query_bytes(c)))
        return fail(MLKV_ERR_INVALID_ARG, "out overlaps blocks");
    if (segments * static_cast<size_t>(n_blocks) >= 1u << 30)   // (sums of two stay within int32)
        return fail(MLKV_ERR_UNSUPPORTED, "%zu listed blocks exceed the int32 indices", segments * n_blocks);
    DeviceGuard guard(c->device);
    if ((rc = prepare_pieces(c, mlkv::kPieceBlocks)) != MLKV_OK)
        return rc;
    static thread_local mlkv::PieceParams p;
    fill_pieces(c, layer, Q, out, seq_lens, p);
    p.blocks = blocks;
    p.n_blocks = n_blocks;
    const auto tiles = [&](int) { return n_blocks; };
    const Cut split = plan_cut(c, {c->b, c->records, false, false, 0, -1}, tiles);
    lay_pieces(c, p, split, tiles);
    return decode_pieces(c, mlkv::kPieceBlocks, p, split, rows64(c), static_cast<cudaStream_t>(cuda_stream));
}

int mlkv_decode_attention_weights(mlkv_cache_t c, int layer, const void *Q, void *out, const int *seq_lens,
                                  const float *weights_in, float *weights_out, void *cuda_stream)
{
    int rc = check_layer(c, layer);
    if (rc != MLKV_OK || (rc = check_queries(c, Q, out)) != MLKV_OK ||
        (rc = check_seq_lens(c, seq_lens)) != MLKV_OK)
        return rc;
    if (weights_out == nullptr || !aligned4(weights_out) || !aligned4(weights_in))
        return fail(MLKV_ERR_INVALID_ARG, "weights must be 4-byte aligned, weights_out non-NULL");
    const size_t bytes = static_cast<size_t>(c->b) * c->g * c->max_seq * 4;
    if ((weights_in != nullptr && weights_in != weights_out && overlap(weights_in, bytes, weights_out, bytes)) ||
        overlap(weights_out, bytes, out, query_bytes(c)) || overlap(weights_out, bytes, Q, query_bytes(c)) ||
        (weights_in != nullptr && overlap(weights_in, bytes, out, query_bytes(c))))
        return fail(MLKV_ERR_INVALID_ARG, "weights_out overlaps another tensor, or out weights_in");
    DeviceGuard guard(c->device);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if ((rc = prepare_pieces(c, mlkv::kPieceWeights)) != MLKV_OK)
        return rc;
    static thread_local mlkv::PieceParams p;
    fill_pieces(c, layer, Q, out, seq_lens, p);
    int longest = 0;
    for (int beta = 0; beta < c->b; ++beta)
        longest = std::max(longest, seq_lens[beta]);
    p.score_stride = (static_cast<long long>(longest) + 63) / 64 * 64;
    if ((rc = scratch(c, static_cast<size_t>(c->b) * c->h * p.score_stride, "scores", stream)) != MLKV_OK)
        return rc;
    p.scores = c->fused_part;
    const auto tiles = [&](int beta) { return mlkv::piece_tiles<mlkv::kPieceWeights>(p, beta); };
    const Cut split = plan_cut(c, {c->b, c->records, true, false, 0, -1}, tiles);
    lay_pieces(c, p, split, tiles);
    mlkv::WeightsParams w;
    w.weights_in = weights_in;
    w.weights_out = weights_out;
    w.max_seq = c->max_seq;
    // (in place, what lies behind the longest sequence stays as it is)
    const long long upto = weights_in == weights_out ? longest : c->max_seq;
    // Positions of a CTA: two rounds of its threads where that still fills the GPU (32 sequences of 8192, 8 KV heads,
    // 176.1 us with 2048, 178.0 with 1024), else one.
    const long long segments = static_cast<long long>(c->b) * c->g;
    w.chunk = segments * ((longest + 2047) / 2048) >= 4LL * c->sm_count ? 2048 : 1024;
    mlkv::plan_weights(c->d, c->G, split.records, &w);
    while (((upto + w.chunk - 1) / w.chunk + w.merge_ctas) * segments > 0x7fffffffLL)
        w.chunk *= 2;
    w.ctas = static_cast<int>((upto + w.chunk - 1) / w.chunk) + w.merge_ctas;
    cudaError_t e = mlkv::launch_pieces(c->d, mlkv::kPieceWeights, rows64(c), rows64(c), p, stream);
    if (e != cudaSuccess)
        return fail_cuda(e, "decode launch");
    e = mlkv::launch_weights(c->d, p, w, split.records, stream);
    return e == cudaSuccess ? MLKV_OK : fail_cuda(e, "weights launch");
}

int mlkv_evict(mlkv_cache_t c, mlkv_cache_t to, int layer, const float *weights_in, float *weights_out,
               const int *seq_lens, const int *keep, int recent, int *kept, int k_max, void *cuda_stream)
{
    int rc = check_layer(c, layer);
    if (rc != MLKV_OK || (rc = mlkv::check_same_model(c, to, "target cache")) != MLKV_OK)
        return rc;
    if (to->b != c->b)
        return fail(MLKV_ERR_MAP, "the target cache holds %d sequences, the cache %d", to->b, c->b);
    if (c->owner[layer] != layer)
        return MLKV_OK;   // its owner's positions are these
    if ((rc = check_seq_lens(c, seq_lens)) != MLKV_OK)
        return rc;
    if (weights_in == nullptr || weights_out == nullptr || kept == nullptr || !aligned4(weights_in) ||
        !aligned4(weights_out) || !aligned4(kept) || keep == nullptr)
        return fail(MLKV_ERR_INVALID_ARG, "weights and kept must be 4-byte aligned; none, nor keep, may be NULL");
    if (recent < 0 || k_max < 1)
        return fail(MLKV_ERR_INVALID_ARG, "recent %d must not be negative, k_max %d be positive", recent, k_max);
    static thread_local mlkv::EvictParams p;
    int longest = 0, rows = 0;
    for (int beta = 0; beta < c->b; ++beta) {
        if (keep[beta] < 1 || keep[beta] < recent)
            return fail(MLKV_ERR_INVALID_ARG, "keep[%d] = %d must be positive and hold the %d newest positions",
                        beta, keep[beta], recent);
        const int n = std::min(keep[beta], seq_lens[beta]);
        if (n > to->max_seq || n > k_max)
            return fail(MLKV_ERR_RANGE, "%d positions of sequence %d exceed k_max %d or the target's %d", n, beta,
                        k_max, to->max_seq);
        p.seq_len[beta] = seq_lens[beta];
        p.keep[beta] = keep[beta];
        longest = std::max(longest, seq_lens[beta]);
        rows = std::max(rows, n);
    }
    const size_t segments = static_cast<size_t>(c->b) * c->g;
    const size_t in = segments * c->max_seq * 4, out = segments * to->max_seq * 4, list = segments * k_max * 4;
    const bool same_w = weights_in == weights_out;
    if (same_w ? c->max_seq != to->max_seq : overlap(weights_in, in, weights_out, out))
        return fail(MLKV_ERR_INVALID_ARG, "weights_out overlaps weights_in, or is it with rows of another length");
    if (overlap(kept, list, weights_in, in) || overlap(kept, list, weights_out, out))
        return fail(MLKV_ERR_INVALID_ARG, "kept overlaps weights");
    p.units = mlkv::evict_units(c->d, rows);
    p.rows = rows;
    if (segments * p.units > 0x7fffffffu || segments > (1u << 24))
        return fail(MLKV_ERR_UNSUPPORTED, "%zu KV heads of %d units exceed a launch", segments, p.units);
    DeviceGuard guard(c->device);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if ((rc = scratch(c, mlkv::evict_flags(static_cast<long long>(segments), p.units), "flags", stream)) != MLKV_OK)
        return rc;
    cudaError_t e = cudaSuccess;
    if (!(c->long_ready & kReadyEvict) && (e = mlkv::prepare_evict()) == cudaSuccess)
        c->long_ready |= kReadyEvict;
    const size_t from_slot = c->cache_bytes / c->m, to_slot = to->cache_bytes / to->m;
    p.src = reinterpret_cast<const __nv_bfloat16 *>(static_cast<char *>(c->cache) + from_slot * c->slot[layer]);
    p.dst = reinterpret_cast<__nv_bfloat16 *>(static_cast<char *>(to->cache) + to_slot * to->slot[layer]);
    p.weights_in = weights_in;
    p.weights_out = weights_out;
    p.kept = kept;
    p.flags = reinterpret_cast<unsigned *>(c->fused_part);
    p.err = c->err;
    p.b = c->b;
    p.g = c->g;
    p.src_seq = c->max_seq;
    p.dst_seq = to->max_seq;
    p.k_max = k_max;
    p.recent = recent;
    p.in_place = c == to || same_w ? 1 : 0;
    p.same = c == to && same_w ? 1 : 0;
    if (e == cudaSuccess)
        e = mlkv::launch_evict(c->d, p, longest, c->sm_count, stream);
    return e == cudaSuccess ? MLKV_OK : fail_cuda(e, "eviction launch");
}

}  // extern "C"
