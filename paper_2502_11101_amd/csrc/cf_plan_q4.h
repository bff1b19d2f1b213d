// The launch plan of the attention over a store in 4 bits: how rows, tokens and splits map to wavefronts and where the partial results
// live in the workspace.  Host arithmetic on the call's sizes alone.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "cachefocus.h"

namespace cf {
namespace q4 {

constexpr int kSoloWaves = 8;       // wavefronts of attn_q4_solo_kernel's workgroups, each with tiles of its own
constexpr int kRowsWaves = 8;       // of attn_q4_rows_kernel's, which share tiles
constexpr int kD = 128;
constexpr int kTile = 32;           // tokens per tile
constexpr int kMaxSplit = 64;
constexpr int kMaxEntries = 256;    // table entries of a query

struct Plan {
    int group;          // query heads per kv head
    int solo;           // attn_q4_solo_kernel (one 16-row block), else attn_q4_rows_kernel
    int halves;         // of the latter: the workgroup's halves have runs of their own
    int runs;           // runs of tiles per workgroup
    int rows_wg;        // rows a workgroup has room for
    int n_rg;           // row groups (workgroups side by side) per (query, kv head)
    int units_per_b, units, nsplit, slots;
    int merge_threads;  // of a workgroup of q4_merge_kernel
    int direct_out;     // one split: the attention kernel writes the output rows itself
    size_t off_ml, off_opart, off_massml, total;
};

inline int64_t plan_tiles(int seg_stride, int64_t max_kv_tokens) { return max_kv_tokens / kTile + seg_stride; }

inline Plan make_plan(int n_q_heads, int n_kv_heads, int batch, int max_tq, int seg_stride, int64_t max_kv_tokens) {
    Plan p;
    p.group = n_q_heads / n_kv_heads;
    const int64_t blocks = ((int64_t)p.group * max_tq + 15) / 16;
    // One block: a wavefront per run and no barriers (one row over 881 tokens x 32 heads 12.1 us, with rows_kernel and the merge that its
    // splits then need 19.0; 32 conversations of 1000 to 5000 tokens 25.4 and 69.2).
    p.solo = blocks <= 1;
    // Up to four: four wavefronts hold all rows, and two such sets stream runs of their own (three blocks x 32 heads over 1680 tokens 27.2 us;
    // with eight wavefronts' room for rows, half of it unused, 31.1: what is left unused costs the merge).
    p.halves = !p.solo && blocks <= 4;
    p.runs = p.solo ? kSoloWaves : p.halves ? 2 : 1;
    p.rows_wg = p.solo ? 16 : 64;
    auto groups = [&](int rows) { return std::max<int64_t>((16 * blocks + rows - 1) / rows, 1); };
    if (blocks > 4) {
        p.rows_wg = 128;
        // More workgroups than CUs: the fewest rounds' worth of work.  A step of a SIMD costs what its two wavefronts do once each, about as much
        // as 1.5 row blocks, and its rows_wg / 64 row blocks.  (64 queries of 384 rows per kv head over 3000 tokens: 284 us with 128 rows, 189 with
        // 192, 225 with 256.)  Fewer workgroups than that are split, and small ones leave fewer partial rows (448 rows x 4 kv heads x 7500
        // tokens, with the merge: 41.0 us with 128 rows, 45.4 with 192, 45.7 with 256).
        int64_t best = 0;
        for (int rows = 256; rows >= 128 && (int64_t)batch * n_kv_heads * groups(128) > 256; rows -= 64) {
            const int64_t rounds = ((int64_t)batch * n_kv_heads * groups(rows) + 255) / 256, cost = rounds * (3 + 2 * rows / 64);
            if (best == 0 || cost < best) { best = cost; p.rows_wg = rows; }
        }
    }
    // (past what the launch takes these are bounds, and the call is refused)
    constexpr int64_t kMost = INT32_MAX;
    const int64_t units = std::min<int64_t>((int64_t)n_kv_heads * groups(p.rows_wg), kMost) * batch;
    p.n_rg = (int)std::min(groups(p.rows_wg), kMost);
    p.units_per_b = (int)std::min((int64_t)n_kv_heads * p.n_rg, kMost);
    p.units = (int)std::min(units, kMost);
    const int64_t tiles = plan_tiles(seg_stride, max_kv_tokens);
    // At most a workgroup per CU (registers leave no room for a second; 512 where one block streams: 32 conversations of 1000 to 5000 tokens 25.4
    // -> 31.8 us, 4 of 24000 to 31000 23.0 -> 31.0), and no split below two tiles per wavefront, which the merge's launch would outweigh (one
    // row over 881 tokens x 32 heads with one tile: 12.2 -> 14.8).
    const int64_t least = p.solo ? 2 * p.runs : 4;
    p.nsplit = (int)std::max<int64_t>(std::min<int64_t>({256 / std::max(p.units, 1), tiles / least, (int64_t)kMaxSplit}), 1);
    p.direct_out = p.nsplit == 1;
    // Few table entries: many threads for each, whose loads are out at once (11 entries 8.2 us, with 256 threads 12.4; 52 10.7 and 17.0).  Many: no more
    // threads than have work (64 queries of 21 entries 9.4 us, with 1024 threads 30.6).  The lines cross between 102 and 164 entries (whole calls with 1024
    // and 256 threads, 16 rows x 4 kv heads: 102 entries 27.4 and 27.8 us, 164 31.3 and 30.1, 336 43.5 and 38.5; 384 rows x 2: 31.2 and 34.2, 37.6 and
    // 36.5, 61.4 and 55.2; 48 rows x 32: 47.5 and 51.0, 64.8 and 64.4, 118 and 116).
    p.merge_threads = (int64_t)batch * seg_stride > 128 ? 256 : 1024;
    p.slots = seg_stride + p.nsplit * p.runs;
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t o = off; off += (bytes + 255) & ~(size_t)255; return o; };
    const size_t rows = (size_t)units * p.nsplit * p.rows_wg;
    p.off_ml = take(rows * 2 * sizeof(float));
    p.off_opart = take(p.direct_out ? 0 : rows * kD * sizeof(float));
    p.off_massml = take((size_t)units * p.slots * p.rows_wg * 2 * sizeof(float));
    p.total = off;
    return p;
}

}  // namespace q4
}  // namespace cf
