// How launches of the operators for long caches are cut, as far as that is arithmetic alone: no CUDA, so that it is
// tested without a GPU.  Internal.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "mlkv.h"

namespace mlkv {

// How the decode over shared prefixes is launched.
struct PrefixPlan {
    int kc;       // key tiles of 128 positions of a unit
    int sms;      // CTAs of the prefix kernel, one an SM
    bool beside;  // the suffixes run beside it on the other SMs, and are merged by a launch of their own
    double us;    // estimated
};

// For `pairs` unit columns (pairs of query tiles times KV heads) over prefixes of n_kt tiles, and suffixes of
// `bytes`: the least estimated time.  Microseconds: a unit's key tile `tile`, its start and end `edges` of them; the
// suffixes at most `rate` bytes a us an SM and `all` in total.  (The prefix kernel is bound by the tensor cores where
// many sequences share one, the suffixes by HBM: side by side, each has what the other leaves.  Not for
// suffixes of less than 16 MB, which the merge's launch outweighs.)  Fitted to eight shapes, each in ten splits: the
// one taken is at most 3% behind the best of them.  128 sequences of 1024, 8 KV heads of 128, over one prefix of
// 32768: 115 us beside 80 SMs of 52 tiles a unit, 147 one after the other.
inline PrefixPlan plan_prefix(const int *n_kt, const int *pairs, int n, int sm_count, int d, double bytes,
                              int max_chunks)
{
    const double tile = d == 64 ? 0.95 : 1.5, edges = 7, rate = 75e3, all = 6.5e6;
    long long work = 0;
    int longest = 1;
    for (int x = 0; x < n; ++x) {
        work += static_cast<long long>(n_kt[x]) * pairs[x];
        if (pairs[x] > 0)
            longest = std::max(longest, n_kt[x]);
    }
    const int least = std::max(1, (longest + max_chunks - 1) / max_chunks);
    PrefixPlan best = {longest, sm_count, false, 1e30};
    // From four rounds of units at most up to whole prefixes, which are tried in any case: of many sequences or KV
    // heads a unit of a whole prefix may be more rounds than that.
    for (int kc = static_cast<int>(std::clamp<long long>(work / (4LL * sm_count), least, longest));;
         kc = std::min(longest, kc + (kc + 15) / 16)) {
        long long units = 0;
        for (int x = 0; x < n; ++x)
            units += static_cast<long long>((n_kt[x] + kc - 1) / kc) * pairs[x];
        for (int rounds = 1; rounds <= 8; ++rounds) {   // of the units, on as many SMs as it takes
            const int sms = static_cast<int>(std::min<long long>(sm_count, (units + rounds - 1) / rounds));
            const double t = static_cast<double>((units + sms - 1) / sms) * (kc + edges) * tile;
            const double one = (bytes < 16e6 ? 7 : 15) + t + bytes / all;
            if (one < best.us)
                best = {kc, sms, false, one};
            const double beside =
                13 + t + std::max(0.0, bytes - t * std::min(all, rate * (sm_count - sms))) / all;
            if (sm_count - sms >= 8 && bytes >= 16e6 && beside < best.us)
                best = {kc, sms, true, beside};
        }
        if (kc == longest)
            break;
    }
    return best;
}

// The query blocks of b prompts, those that see the most key blocks first, then by sequence: visit(beta, qb) for block
// qb of blocks[beta], behind pre[beta] key blocks of a prefix (NULL: none anywhere).  Stops where visit returns false.
// With prefixes the sequences enter by the last key block that they see and leave behind their first query block, so
// that the host's work is the prompts', however far their prefixes reach (1024 prompts of two blocks behind a million
// positions, 17 ms if every key block is walked through).
template <typename Visit>
inline bool for_query_blocks(int b, const int *blocks, const int *pre, const Visit &visit)
{
    if (pre == nullptr) {
        const int most = *std::max_element(blocks, blocks + b);
        for (int qb = most - 1; qb >= 0; --qb)
            for (int beta = 0; beta < b; ++beta)
                if (qb < blocks[beta] && !visit(beta, qb))
                    return false;
        return true;
    }
    uint16_t order[MLKV_MAX_BATCH], live[MLKV_MAX_BATCH];   // by last key block, falling; those under way, by number
    for (int beta = 0; beta < b; ++beta)
        order[beta] = static_cast<uint16_t>(beta);
    const auto last = [&](int beta) { return pre[beta] + blocks[beta] - 1; };
    std::sort(order, order + b, [&](int x, int y) { return last(x) != last(y) ? last(x) > last(y) : x < y; });
    int n_live = 0, seen = 0;
    for (int next = 0; next < b || n_live > 0; --seen) {
        if (n_live == 0)
            seen = last(order[next]);
        const int before = n_live;
        while (next < b && last(order[next]) == seen)
            live[n_live++] = order[next++];
        if (before > 0 && n_live > before)
            std::inplace_merge(live, live + before, live + n_live);
        for (int i = 0; i < n_live; ++i)
            if (!visit(static_cast<int>(live[i]), seen - pre[live[i]]))
                return false;
        n_live = static_cast<int>(std::remove_if(live, live + n_live, [&](int x) { return pre[x] == seen; }) - live);
    }
    return true;
}

}  // namespace mlkv
