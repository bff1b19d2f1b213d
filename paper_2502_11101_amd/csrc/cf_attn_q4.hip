// Prefill and decode attention over a cache store in 4 bits for gfx950 (head_dim 128, 16-bit queries and outputs).
//
// A stored key or value row is 128 codes of four bits and four scale bytes (32 channels each).  What is moved to other positions is the query
// and not the keys: (R_delta k) . q = k . (R_-delta q), once per segment instead of once per key (Eq. 5), and the keys stay exact.
// Scores.  The turned query, scaled by a power of two of its row, is split into two fp16 terms (22 bits); the keys, unpacked to fp16, are exact (at most two
// significant bits and an exponent inside fp16's), so that scores are right to fp32's accuracy on v_mfma_f32_16x16x32_f16.  (The scaled
// 4-bit instruction, v_mfma_scale_f32_16x16x128_f8f6f4, takes the codes as they lie in memory against a query of e4m3 terms at the same matrix
// cycles, but sums its 128 products with an error of up to 2^-13 of the largest one: attention masses were off by 2e-6 to 5e-6, and with an fp16 term
// and one e4m3 term on that instruction by 7e-7 to 1.1e-6.)
// Values are unpacked to fp16, staged in LDS and read transposed; probabilities are rounded to fp16 (2^-11, see kLift), sums, maxima and accumulators
// are fp32.  Tiles with a scale outside fp16's exponents are left to a second pass over the run, in bf16: queries of three terms,
// probabilities as value and remainder.
//
// Work: the rows that share a kv head (row m = t * group + head) are cut into 16-row blocks.
//   * One block (decode steps): attn_q4_solo_kernel, each of eight wavefronts streams a run of 32-token tiles of its own; they meet in LDS at the end.
//   * More: attn_q4_rows_kernel, eight wavefronts that share the tiles that they stage together.
// Splits (workgroups of the same rows) leave fp32 partial rows that q4_merge_kernel merges; it also reduces the (reference, sum) pairs
// that the wavefronts leave per row and segment where masses are wanted.
#include "cf_attn_tile.h"
#include "cf_plan_q4.h"

namespace cf {
namespace q4 {

using attn::build_reg_table;
using attn::build_table;
using attn::f32x4;
using attn::load_query_head;
using attn::Mma;
using attn::QueryHead;
using attn::RegSegTable;
using attn::rope_cos_sin_fast;
using attn::SegTable;
using attn::short4v;
using attn::Tile;
using attn::wave_lds_order;

namespace {

constexpr int kSoloThreads = kSoloWaves * kWave, kRowsThreads = kRowsWaves * kWave, kMergeThreads = 1024;
constexpr int kMassRows = 2048;
constexpr int kKRow = 272, kVRow = 288;              // bytes per token of a staged tile
constexpr int kKTile = kTile * kKRow, kVTile = kTile * kVRow;
constexpr int kRowBytes = 64;                        // codes of a row
constexpr int kQRow = 272;                           // bytes per row of queries in LDS
// Probabilities that are rounded to fp16 are relative to a reference kLift below a row's maximum in the exponent: the largest are 2^8, those down to 2^-22
// of it keep eleven bits, those below a step of 2^-32 of it.  (Relative to the maximum itself: 2^-14 and 2^-24; of thousands of tokens 16 nats below a
// dominant one 6 % were lost, from 17.5 nats on everything.)  The reference stays where it is until a lane's eight add up to more than
// kLiftLimit, so that each is a number of fp16: room for 2^8 above it, as kProbLimit leaves without a lift.  (A lift of 11 with room for 2^5: 64 queries of
// 384 rows x 2 heads 1.5 % slower, the reference moves more often.)
constexpr int kLift = 8;
constexpr float kLiftLimit = 65504.f;
// Tiles in bf16 may have values of up to the type's largest, and bf16 probabilities any exponent: there the reference is kDrop above the maximum, so that
// the accumulators, sums over thousands of tokens before they are divided, stay finite.  (No further above it: products of values next to nothing come
// near fp32's smallest numbers; 2^-24 was more than values of 2^-112 bear.)
constexpr int kDrop = -12;
constexpr float kDropLimit = attn::kProbLimit / (1 << -kDrop);
template <int DT> constexpr int kOwnLift = DT == CF_BF16 ? kDrop : kLift;

// run i of a list of `total` tiles owns [total*i/n, total*(i+1)/n) (n at most 512, so that shorter lists need no 64-bit division)
__device__ __forceinline__ int run_begin(int total, int n, int i) {
    if (total < (1 << 22)) return (int)div_exact((unsigned)(total * i), (unsigned)n);
    return (int)((int64_t)total * i / n);
}
// the run that owns tile x
__device__ __forceinline__ int run_of(int total, int n, int x) {
    if (total < (1 << 22)) return (int)div_exact((unsigned)((x + 1) * n - 1), (unsigned)total);
    return (int)((((int64_t)x + 1) * n - 1) / total);
}

// The arguments that a kernel needs on its way to its first tile, asked for at once (the compiler would load each where it is first used, a round
// trip every time).
__device__ __forceinline__ void ask_for_arguments(const AttnArgs& a, const Plan& p, const Scales& s) {
    const void *p0 = a.q, *p1 = a.q_off, *p2 = a.q_new_start, *p3 = a.k_store, *p4 = a.v_store, *p5 = s.k, *p6 = s.v, *p7 = a.segs, *p8 = a.n_seg,
               *p9 = a.workspace, *p10 = a.mass, *p11 = a.k_self;
    asm volatile("" ::"s"(p0), "s"(p1), "s"(p2), "s"(p3), "s"(p4), "s"(p5), "s"(p6), "s"(p7), "s"(p8), "s"(p9), "s"(p10), "s"(p11), "s"(a.n_store_tokens),
                 "s"(a.seg_stride), "s"(a.batch), "s"(a.max_tq), "s"(a.n_q_heads), "s"(a.n_kv_heads), "s"(a.q_stored_start), "s"(a.store_ts),
                 "s"(a.store_hs), "s"(a.max_positions), "s"(p.group), "s"(p.n_rg), "s"(p.nsplit), "s"(p.slots));
}

// A query's table in LDS, laid out for the walk: where a segment's tiles end, by kind (0: of the other kind, or empty), and its fields side by side.
struct RunTable {
    int4 row[kMaxEntries];      // first tile, past the last tile, visible tokens, shift
    int64_t tok[kMaxEntries];   // first token in its tensor
    int store_end[kMaxEntries], own_end[kMaxEntries];
    int n, total;
};
// All threads of a workgroup of at least kMaxEntries call this, and pass a barrier before they use the table or what tmp was made from.
__device__ __forceinline__ void build_run_table(const AttnArgs& a, const QueryHead& qh, RunTable* t, SegTable* tmp) {
    const int tid = threadIdx.x;
    auto put = [&](int s, int first, int end, int vis, int delta, int self, int64_t tok) __attribute__((always_inline)) {
        t->row[s] = make_int4(first, end, vis, delta);
        t->tok[s] = tok;
        t->store_end[s] = !self && vis > 0 ? end : 0;
        t->own_end[s] = self && vis > 0 ? end : 0;
    };
    if (a.seg_stride <= kWave) {                     // the first wavefront's registers do
        if (tid < kWave) {
            const RegSegTable r = build_reg_table(a, qh, tid, kTile);
            put(tid, r.t0, r.t1, tid < r.n ? r.vis : 0, r.delta, r.self, r.tok);
            if (tid == 0) { t->n = r.n; t->total = r.total; }
        }
    } else {
        build_table(a, qh, tmp, kTile);
        const int n = tmp->n;
        if (tid < n) put(tid, tmp->tile0[tid], tmp->tile0[tid + 1], tmp->vis[tid], tmp->delta[tid], tmp->self[tid], tmp->tok[tid]);
        else if (tid < kMaxEntries) put(tid, 0, 0, 0, 0, 0, 0);
        if (tid == 0) { t->n = n; t->total = tmp->tile0[n]; }
    }
}

// The first segment of a kind (of the own block, or of the store) whose tiles reach past tile x; -1: none.  `prev`: a segment that is not behind it.
template <bool OWN>
__device__ __forceinline__ int find_kind(const RunTable& t, int x, int lane, int prev) {
    for (int s0 = prev < 0 ? 0 : prev & ~(kWave - 1); s0 < t.n; s0 += kWave) {
        const uint64_t hit = __ballot((OWN ? t.own_end : t.store_end)[s0 + lane] > x);
        if (hit) return s0 + __builtin_ctzll(hit);
    }
    return -1;
}
template <bool OWN>
__device__ __forceinline__ int find_kind(const RegSegTable& t, int x, int lane, int) {
    const uint64_t hit = __ballot(lane < t.n && t.t1 > x && (t.self != 0) == OWN && t.vis > 0);
    return hit ? __builtin_ctzll(hit) : -1;
}
__device__ __forceinline__ int first_tile(const RunTable& t, int s) { return __builtin_amdgcn_readfirstlane(t.row[s].x); }
__device__ __forceinline__ int first_tile(const RegSegTable& t, int s) { return __builtin_amdgcn_readlane(t.t0, s); }
struct SegFields { int first, end, vis, delta; int64_t tok; };
__device__ __forceinline__ int64_t scalar64(int64_t x) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)((uint64_t)x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ SegFields fields(const RunTable& t, int s) {
    auto scalar = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    const int4 row = t.row[s];
    const int64_t tok = t.tok[s];
    return {scalar(row.x), scalar(row.y), scalar(row.z), scalar(row.w), scalar64(tok)};
}
__device__ __forceinline__ SegFields fields(const RegSegTable& t, int s) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)t.tok, s), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)t.tok >> 32), s);
    return {__builtin_amdgcn_readlane(t.t0, s), __builtin_amdgcn_readlane(t.t1, s), __builtin_amdgcn_readlane(t.vis, s), __builtin_amdgcn_readlane(t.delta, s),
            (int64_t)((uint64_t)hi << 32 | lo)};
}
// whether a run holds tiles of the kind
template <bool OWN, class Table>
__device__ __forceinline__ bool holds(const Table& t, int begin, int end, int lane) {
    const int s = begin < end ? find_kind<OWN>(t, begin, lane, -1) : -1;
    return s >= 0 && first_tile(t, s) < end;
}

// Walks the tiles of a run that lie in the store, or (OWN) in the own block.
template <bool OWN>
struct RunWalk {
    int next_tile, t_end;
    int c_seg = -1, c_first = 0, c_end = 0, c_vis = 0, c_delta = 0;
    int64_t c_tok = 0;          // first token of the cached segment in its tensor

    __device__ __forceinline__ RunWalk(int begin, int end) : next_tile(begin), t_end(end) {}

    // to the next tile of the kind, or to the end
    template <class Table>
    __device__ __forceinline__ void settle(const Table& tbl, int lane) {
        if (next_tile >= t_end || next_tile < c_end) return;
        const int s = find_kind<OWN>(tbl, next_tile, lane, c_seg);
        if (s < 0) {
            next_tile = t_end;
            return;
        }
        const SegFields f = fields(tbl, s);
        c_seg = s;
        c_first = f.first;
        c_end = f.end;
        c_vis = f.vis;
        c_delta = f.delta;
        c_tok = f.tok;
        next_tile = max(next_tile, c_first);
    }
    // The next tile, or one with ntok == 0 when none is left.
    template <class Table>
    __device__ __forceinline__ Tile next(const Table& tbl, int lane) {
        Tile d;
        d.seg = 0; d.tok0 = 0; d.ntok = 0; d.delta = 0; d.self = 0;
        settle(tbl, lane);
        if (next_tile < t_end) {
            d.seg = c_seg;
            d.tok0 = (next_tile - c_first) * kTile;
            d.ntok = min(kTile, c_vis - d.tok0);
            d.delta = c_delta;
            ++next_tile;
        }
        return d;
    }
    template <class Table>
    __device__ __forceinline__ void skip(const Table& tbl, int lane) {
        settle(tbl, lane);
        ++next_tile;
    }
};

// 8 codes (channels c .. c+7) with their scale as eight 16-bit floats
template <int DT>
__device__ __forceinline__ uint4 unpack8(uint32_t codes, float scale) {
    if constexpr (DT == CF_F16)
        return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 0)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 1)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 2)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 3)));
    else
        return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3)));
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }
// exponents at which every code is a number of fp16: 2^-23 .. 2^13
__device__ __forceinline__ bool fits_f16(uint32_t byte) { return byte - 104u <= 36u; }

// A lane's part of row li of a 16-row block of queries: channels 16 lg .. + 15 and 64 + 16 lg .. + 15, as they lie in memory.
struct QueryPart { uint4 w[4]; };
__device__ __forceinline__ QueryPart load_query(const uint16_t* qp, bool valid, int lg) {
    QueryPart q;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        q.w[i] = valid ? *reinterpret_cast<const uint4*>(qp + 16 * lg + 64 * (i >> 1) + 8 * (i & 1)) : make_uint4(0, 0, 0, 0);
    return q;
}
// Its channels 4n .. 4n + 3 of either half (a, b), turned by -delta.  cs: (cos, sin) of delta's 64 angles.
template <int DT, int PAIRING>
__device__ __forceinline__ void turn4(const QueryPart& q, int n, const float2* cs, int lg, float (&a)[4], float (&b)[4]) {
    const uint4 wa = q.w[n >> 1], wb = q.w[2 + (n >> 1)];
    const uint32_t ua[2] = {n & 1 ? wa.z : wa.x, n & 1 ? wa.w : wa.y}, ub[2] = {n & 1 ? wb.z : wb.x, n & 1 ? wb.w : wb.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = i & 1 ? Mma<DT>::hi(ua[i >> 1]) : Mma<DT>::lo(ua[i >> 1]);
        b[i] = i & 1 ? Mma<DT>::hi(ub[i >> 1]) : Mma<DT>::lo(ub[i >> 1]);
    }
    if constexpr (PAIRING == CF_ROPE_HALF) {         // slice m: channels m, m + 64
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 c = cs[16 * lg + 4 * n + i];
            const float x = a[i], y = b[i];
            a[i] = x * c.x + y * c.y;
            b[i] = y * c.x - x * c.y;
        }
    } else {                                         // slice m: channels 2m, 2m + 1
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float2 c = cs[8 * lg + 2 * n + i], d = cs[32 + 8 * lg + 2 * n + i];
            const float x = a[2 * i], y = a[2 * i + 1], u = b[2 * i], w = b[2 * i + 1];
            a[2 * i] = x * c.x + y * c.y;
            a[2 * i + 1] = y * c.x - x * c.y;
            b[2 * i] = u * d.x + w * d.y;
            b[2 * i + 1] = w * d.x - u * d.y;
        }
    }
}

// The bits of the largest magnitude among a lane's channels, but for those that are not finite.
template <int DT>
__device__ __forceinline__ uint32_t largest(const QueryPart& q) {
    constexpr uint32_t kInf = DT == CF_BF16 ? 0x7f80u : 0x7c00u;
    uint32_t top = 0;
    auto take = [&](uint32_t x) { top = max(top, x < kInf ? x : 0u); };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t u[4] = {q.w[i].x, q.w[i].y, q.w[i].z, q.w[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            take(u[j] & 0x7fffu);
            take(u[j] >> 16 & 0x7fffu);
        }
    }
    return top;
}
// The exponent byte of the power of two that a row of queries is scaled down by: its largest channel comes to between 1 and 2.
template <int DT>
__device__ __forceinline__ int row_scale(const QueryPart& q) {
    uint32_t top = largest<DT>(q);
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    return min(max((int)(__float_as_uint(Mma<DT>::lo(top)) >> 23), 27), 253);
}
// The softmax scale (times log2 e) as a power of two, which multiplies scores, and a factor of the angles' cos and sin.  Scores times a power of two are
// exact, so that the largest one less the reference made of it is zero whatever its size (times anything else it is off by a rounding of the
// score, which exp2 of scores past 2^24 does not survive).
__device__ __forceinline__ float scale_power(float scale_log2e) { return __uint_as_float(__float_as_uint(scale_log2e) & 0x7f800000u); }
__device__ __forceinline__ float scale_factor(float scale_log2e) { return __uint_as_float((__float_as_uint(scale_log2e) & 0x807fffffu) | 0x3f800000u); }
// What a row's scores are in units of, from the exponent byte of its own power of two.  (Not zero, however small the softmax scale: a masked score is minus
// infinity times this.)
__device__ __forceinline__ float score_unit(float scale_log2e, int scale) {
    return fmaxf(scale_power(scale_log2e) * __uint_as_float((uint32_t)scale << 23), 0x1p-126f);
}
__device__ __forceinline__ float scale_down(int scale) { return __uint_as_float((uint32_t)(254 - scale) << 23); }
// The row in its own type, scaled: exact but for channels 2^-14 (fp16) of the largest and less, which keep what lies above 2^-25 of it.  (Every row by its
// own: scaled together, a row with a channel 2^20 larger would take the bits of those beside it.)
template <int DT>
__device__ __forceinline__ QueryPart scaled(const QueryPart& q, int scale) {
    const float down = scale_down(scale);
    QueryPart r;
    auto two = [&](uint32_t u) { return Mma<DT>::pack(Mma<DT>::lo(u) * down, Mma<DT>::hi(u) * down); };
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = make_uint4(two(q.w[i].x), two(q.w[i].y), two(q.w[i].z), two(q.w[i].w));
    return r;
}

// two floats as 16-bit values and what is left of them
template <int DT>
__device__ __forceinline__ void split2(float x, float y, uint32_t& hi, uint32_t& lo) {
    hi = Mma<DT>::pack(x, y);
    lo = Mma<DT>::pack(fmaf(Mma<DT>::lo(hi), -1.f, x), fmaf(Mma<DT>::hi(hi), -1.f, y));
}
template <int DT>
__device__ __forceinline__ void split8(const float (&v)[8], uint4& hi, uint4& lo) {
    split2<DT>(v[0], v[1], hi.x, lo.x);
    split2<DT>(v[2], v[3], hi.y, lo.y);
    split2<DT>(v[4], v[5], hi.z, lo.z);
    split2<DT>(v[6], v[7], hi.w, lo.w);
}

// A 16-row block of turned queries as matrix operands of type OT, value and remainder.  A matrix product does not mind the order of its channels as
// long as both sides have the same: operand c of a lane holds channels 16 lg + 8 c .. + 7 (c < 2) or 64 + 16 lg + 8 (c - 2) .. + 7, which are those
// that the lane turns.
struct Parts { uint4 hi[4], lo[4]; };
template <int DT, int PAIRING, int OT>
__device__ __forceinline__ Parts to_parts(const QueryPart& q, const float2* cs, int lg) {
    Parts r;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        float a0[4], b0[4], a1[4], b1[4];
        turn4<DT, PAIRING>(q, 2 * c, cs, lg, a0, b0);
        turn4<DT, PAIRING>(q, 2 * c + 1, cs, lg, a1, b1);
        const float va[8] = {a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]};
        const float vb[8] = {b0[0], b0[1], b0[2], b0[3], b1[0], b1[1], b1[2], b1[3]};
        split8<OT>(va, r.hi[c], r.lo[c]);
        split8<OT>(vb, r.hi[2 + c], r.lo[2 + c]);
        __builtin_amdgcn_sched_barrier(0);           // few floats at a time
    }
    return r;
}

// eight 16-bit values, zeros where they are not finite; any: whether there were some
template <int DT>
__device__ __forceinline__ uint4 finite8(uint4 v, bool& any) {
    constexpr uint32_t kMask = DT == CF_BF16 ? 0x7f80u : 0x7c00u;
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool lo = (w[i] & kMask) == kMask, hi = (w[i] & kMask << 16) == kMask << 16;
        any = any || lo || hi;
        w[i] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A staged tile of values, transposed: operand db holds channels 16 db .. + 15.
struct Values { uint4 f[8]; };
__device__ __forceinline__ Values load_values(const unsigned char* v_read) {
    Values v;
#pragma unroll
    for (int db = 0; db < 8; ++db) {
        const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)(v_read + 32 * db));
        const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)(v_read + 32 * db + 16 * kVRow));
        const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
        v.f[db] = make_uint4(l2.x, l2.y, h2.x, h2.y);
    }
    return v;
}

// ---------------------------------------------------------------------------------------------
// What a wavefront accumulates for its NRB 16-row blocks, and what it needs to go on: lane (li, lg) holds, for row li of each block, the output
// channels 16 db + 4 lg + r, the reference maximum and the sums over the tokens that it has seen (whole call and current segment).
template <int NRB>
struct Rows {
    f32x4 acc[NRB][8];
    float m_run[NRB], l_run[NRB], seg_l[NRB];
    int trow[NRB], qrow[NRB];   // place in the own block (-1: no row); row of q and out, counted from the query's first
    int cur_seg;

    // the rows from `row0` on of kv head `hkv`, of which the query has n_rows
    __device__ __forceinline__ void begin(int row0, int n_rows, int group, int n_q_heads, int hkv, int li) {
        cur_seg = -1;
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
#pragma unroll
            for (int db = 0; db < 8; ++db) acc[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
            m_run[rb] = -INFINITY;
            l_run[rb] = seg_l[rb] = 0.f;
            const int m = row0 + 16 * rb + li;
            const bool valid = m < n_rows;
            const int t = valid ? (int)div_exact((unsigned)m, (unsigned)group) : 0, g = valid ? m - t * group : 0;
            trow[rb] = valid ? t : -1;
            qrow[rb] = t * n_q_heads + hkv * group + g;
        }
    }
    // One place for the accumulators: across a branch that scales them the compiler would otherwise keep a copy for either way (at two
    // row blocks that spilled 200 bytes a lane).
    __device__ __forceinline__ void pin() {
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
            for (int db = 0; db < 8; ++db) asm volatile("" : "+v"(acc[rb][db]));
    }
    // Online softmax (exp2 domain) of scores sc, in units of mul(block), against a stale row maximum less LIFT: probabilities pv; see kLift.
    template <int LIFT, class F>
    __device__ __forceinline__ void softmax(f32x4 (&sc)[NRB][2], F mul, float (&pv)[NRB][8]) {
        constexpr float kLimit = LIFT > 0 ? kLiftLimit : kDropLimit;
        float lsum[NRB];
        auto probabilities = [&](int rb) __attribute__((always_inline)) {
            const float m_safe = m_run[rb] == -INFINITY ? 0.f : m_run[rb];
            lsum[rb] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                pv[rb][e] = __builtin_amdgcn_exp2f(fmaf(sc[rb][e >> 2][e & 3], mul(rb), -m_safe));
                lsum[rb] += pv[rb][e];
            }
        };
        bool off = false;
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            probabilities(rb);
            off = off || !(lsum[rb] <= kLimit) || m_run[rb] == -INFINITY;
        }
        if (__any(off)) {
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) {
                float mloc = -INFINITY;
#pragma unroll
                for (int e = 0; e < 8; ++e) mloc = fmaxf(mloc, sc[rb][e >> 2][e & 3]);
                mloc *= mul(rb);                     // > 0: max commutes with it
                mloc = fmaxf(mloc, __shfl_xor(mloc, 16));
                mloc = fmaxf(mloc, __shfl_xor(mloc, 32));
                const float ref = mloc - LIFT;       // (a step of scores past 2^27 may come to more than the lift)
                mloc = LIFT > 0 && mloc - ref > LIFT ? mloc : ref;
                const float m_new = fmaxf(m_run[rb], mloc);
                const float alpha = __builtin_amdgcn_exp2f(m_run[rb] - (m_new == -INFINITY ? 0.f : m_new));
#pragma unroll
                for (int db = 0; db < 8; ++db) acc[rb][db] *= alpha;
                l_run[rb] *= alpha;
                seg_l[rb] *= alpha;
                m_run[rb] = m_new;
                probabilities(rb);
            }
        }
        pin();
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            l_run[rb] += lsum[rb];
            seg_l[rb] += lsum[rb];
        }
    }
    // From kLift to kDrop.
    __device__ __forceinline__ void lower() {
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            const float m_new = m_run[rb] + (kLift - kDrop), f = m_run[rb] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[rb] - m_new);
#pragma unroll
            for (int db = 0; db < 8; ++db) acc[rb][db] *= f;
            l_run[rb] *= f;
            seg_l[rb] *= f;
            m_run[rb] = m_new;
        }
        pin();
    }
    // O^T += V^T P^T, V of the type VT.  EXACT: P as value and remainder.
    template <int VT, bool EXACT>
    __device__ __forceinline__ void weigh(const Values& v, const float (&pv)[NRB][8]) {
        uint4 ph[NRB], pl[NRB];
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) split8<VT>(pv[rb], ph[rb], pl[rb]);
#pragma unroll
        for (int db = 0; db < 8; ++db) {
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) {
                if constexpr (EXACT) acc[rb][db] = Mma<VT>::run(v.f[db], pl[rb], acc[rb][db]);
                acc[rb][db] = Mma<VT>::run(v.f[db], ph[rb], acc[rb][db]);
            }
        }
    }
    // (reference, sum) per row of the segment that ends here, to its slot; `again`: added to what the slot holds, whose reference is not larger
    __device__ __forceinline__ void emit(float2* massml, int rows_wg, int ss, bool again, int li, int lg) {
        if (cur_seg < 0 || massml == nullptr) return;
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            float tot = seg_l[rb] + __shfl_xor(seg_l[rb], 16);
            tot += __shfl_xor(tot, 32);
            if (lg == 0) {
                float2* slot = massml + (int64_t)(cur_seg + ss) * rows_wg + 16 * rb + li;
                if (again && slot->x != -INFINITY) tot += slot->y * __builtin_amdgcn_exp2f(slot->x - m_run[rb]);
                *slot = make_float2(m_run[rb], tot);
            }
        }
    }
    __device__ __forceinline__ void enter(int seg, float2* massml, int rows_wg, int ss, bool again, int li, int lg) {
        if (seg == cur_seg) return;
        emit(massml, rows_wg, ss, again, li, lg);
        cur_seg = seg;
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) seg_l[rb] = 0.f;
    }
    // row sums over the four lane groups
    __device__ __forceinline__ void close() {
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            l_run[rb] += __shfl_xor(l_run[rb], 16);
            l_run[rb] += __shfl_xor(l_run[rb], 32);
        }
    }
};

// A buffer of `range` bytes from base + off on; reads past it give zero.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* base, int64_t off, int range) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(base) + off), 0, range, 0x00020000);
}

// A tile of the store for a wavefront on its own: of token 16 tb + li the key channels 16 lg .. + 15 and 64 + 16 lg .. + 15 with all four scales,
// and 32 value channels from 32 lg on.
struct TileRegs { uint2 k[2][2]; uint4 v[2]; uint32_t ks[2], vs[2]; };
__device__ __forceinline__ void load_tile(const AttnArgs& a, const Scales& s, const Tile& d, int64_t seg_tok, int hkv, int li, int lg, TileRegs& r) {
    const int row_bytes = (int)(a.store_ts >> 1), scale_bytes = (int)(a.store_ts >> 5);
    // rows past a ragged tile's end, and everything where no tile is left, lie past the range and read as zero
    const bool any = d.ntok > 0;
    const int64_t at = any ? (seg_tok + d.tok0) * a.store_ts + (int64_t)hkv * a.store_hs : 0;
    const int codes = any ? (d.ntok - 1) * row_bytes + kRowBytes : 0, scales = any ? (d.ntok - 1) * scale_bytes + 4 : 0;
    const auto rk = buffer(a.k_store, at >> 1, codes), rv = buffer(a.v_store, at >> 1, codes);
    const auto sk = buffer(s.k, at >> 5, scales), sv = buffer(s.v, at >> 5, scales);
#pragma unroll
    for (int tb = 0; tb < 2; ++tb) {
        const int off = (16 * tb + li) * row_bytes, soff = (16 * tb + li) * scale_bytes;
        r.k[tb][0] = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(rk, off + 8 * lg, 0, 0));
        r.k[tb][1] = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(rk, off + 8 * lg + 32, 0, 0));
        r.v[tb] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rv, off + 16 * lg, 0, 0));
        r.ks[tb] = __builtin_amdgcn_raw_buffer_load_b32(sk, soff, 0, 0);
        r.vs[tb] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(sv, soff + lg, 0, 0);
    }
}
// operand c of the keys 16 tb .. + 15 (see Parts)
template <int DT>
__device__ __forceinline__ uint4 key_operand(const TileRegs& r, int tb, int c, int lg) {
    const uint2 w = r.k[tb][c >> 1];
    return unpack8<DT>(c & 1 ? w.y : w.x, scale_of(__builtin_amdgcn_ubfe(r.ks[tb], 16 * (c >> 1) + 8 * (lg >> 1), 8)));
}
__device__ __forceinline__ bool tile_fits(const TileRegs& r, int ntok, int li, int lg) {
    bool fits = true;
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
        fits = fits && ((fits_f16(__builtin_amdgcn_ubfe(r.ks[tb], 8 * lg, 8)) && fits_f16(r.vs[tb])) || 16 * tb + li >= ntok);
    return __all(fits);
}
__device__ __forceinline__ void stage_values(unsigned char* to, uint4 codes, float scale) {
    reinterpret_cast<uint4*>(to)[0] = unpack8<CF_F16>(codes.x, scale);
    reinterpret_cast<uint4*>(to)[1] = unpack8<CF_F16>(codes.y, scale);
    reinterpret_cast<uint4*>(to)[2] = unpack8<CF_F16>(codes.z, scale);
    reinterpret_cast<uint4*>(to)[3] = unpack8<CF_F16>(codes.w, scale);
}

// What the passes of a wavefront on its own need of the kernel around them.
struct WavePlace {
    int li, lg, hkv, rows_wg, ss;
    int t_begin, t_end;         // its run of tiles
    int64_t q_first;            // the query's first row in q and out, in elements
    double my_freq;             // of slice `lane`
    float2* cs;                 // 64 entries of LDS
    unsigned char* v_lds;       // kVTile bytes of LDS
    float2* massml;             // slots of its rows, or NULL
};

// cos and sin of an angle of the query's turn, with the softmax scale's factor
__device__ __forceinline__ float2 turn_angle(const AttnArgs& a, int delta, double freq) {
    const float2 c = rope_cos_sin_fast(delta, freq);
    const float f = scale_factor(a.scale_log2e);
    return make_float2(c.x * f, c.y * f);
}
// those of delta's 64 angles to LDS
__device__ __forceinline__ void put_angles(const AttnArgs& a, float2* cs, int lane, int delta, double my_freq) {
    wave_lds_order();
    cs[lane] = turn_angle(a, delta, my_freq);
    wave_lds_order();
}

template <int NRB>
__device__ __forceinline__ QueryPart query_part(const AttnArgs& a, int64_t q_first, const Rows<NRB>& st, int rb, int lg) {
    int row = st.qrow[rb];
    asm volatile("" : "+v"(row));                    // its addresses are worked out anew, not kept through the loops
    return load_query(static_cast<const uint16_t*>(a.q) + q_first + (int64_t)row * kD, st.trow[rb] >= 0, lg);
}

// The scale of a row of queries in the second pass, where keys have any scale: between its largest channel and 2^-9 there is room for keys
// up to 2^127 and down to 2^-117.
constexpr int kOddScale = 9;

// The second pass over a run: the tiles whose scales do not fit fp16, in bf16: queries of three terms, probabilities as value and remainder.
// The segments' slots hold sums already.
template <int DT, int PAIRING, int NRB, class Table>
__device__ __forceinline__ void odd_tiles(const AttnArgs& a, const Scales& s, const Table& tbl, const WavePlace& w, Rows<NRB>& st) {
    st.emit(w.massml, w.rows_wg, w.ss, false, w.li, w.lg);
    st.cur_seg = -1;
    const int lane = 16 * w.lg + w.li;
    RunWalk<false> walk(w.t_begin, w.t_end);
    for (;;) {
        const Tile d = walk.next(tbl, lane);
        if (d.ntok <= 0) break;
        TileRegs r;
        load_tile(a, s, d, walk.c_tok, w.hkv, w.li, w.lg, r);
        if (tile_fits(r, d.ntok, w.li, w.lg)) continue;
        st.enter(d.seg, w.massml, w.rows_wg, w.ss, true, w.li, w.lg);
        put_angles(a, w.cs, lane, d.delta, w.my_freq);
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            uint4* const to = reinterpret_cast<uint4*>(w.v_lds + (16 * tb + w.li) * kVRow + 64 * w.lg);
            const float scale = scale_of(r.vs[tb]);
            to[0] = unpack8<CF_BF16>(r.v[tb].x, scale);
            to[1] = unpack8<CF_BF16>(r.v[tb].y, scale);
            to[2] = unpack8<CF_BF16>(r.v[tb].z, scale);
            to[3] = unpack8<CF_BF16>(r.v[tb].w, scale);
        }
        wave_lds_order();
        f32x4 sc[NRB][2];
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            const QueryPart q = query_part(a, w.q_first, st, rb, w.lg);
            const int scale = min(row_scale<DT>(q) + kOddScale, 253);
            const float down = scale_down(scale);
            sc[rb][0] = sc[rb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 2; ++c) {            // channels 8c .. 8c + 7 of either half
                float v[4][4];
                turn4<DT, PAIRING>(q, 2 * c, w.cs, w.lg, v[0], v[2]);
                turn4<DT, PAIRING>(q, 2 * c + 1, w.cs, w.lg, v[1], v[3]);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint4 term[3];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float x = v[2 * h + (i >> 1)][2 * (i & 1)] * down, y = v[2 * h + (i >> 1)][2 * (i & 1) + 1] * down;
#pragma unroll
                        for (int k = 0; k < 3; ++k) {
                            const uint32_t pair = Mma<CF_BF16>::pack(x, y);
                            x -= Mma<CF_BF16>::lo(pair);
                            y -= Mma<CF_BF16>::hi(pair);
                            reinterpret_cast<uint32_t*>(&term[k])[i] = pair;
                        }
                    }
#pragma unroll
                    for (int tb = 0; tb < 2; ++tb) {
                        const uint4 kf = key_operand<CF_BF16>(r, tb, 2 * h + c, w.lg);
#pragma unroll
                        for (int k = 2; k >= 0; --k) sc[rb][tb] = Mma<CF_BF16>::run(kf, term[k], sc[rb][tb]);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            const int lim = d.ntok - 4 * w.lg;
            const float up = scale_power(a.scale_log2e) * scale_of((uint32_t)scale);
#pragma unroll
            for (int e = 0; e < 8; ++e) sc[rb][e >> 2][e & 3] = 16 * (e >> 2) + (e & 3) < lim ? sc[rb][e >> 2][e & 3] * up : -INFINITY;
        }
        float pv[NRB][8];
        st.template softmax<kOwnLift<DT>>(sc, [&](int) { return 1.f; }, pv);
        st.template weigh<CF_BF16, true>(load_values(w.v_lds + (4 * w.lg + (w.li >> 2)) * kVRow + 8 * (w.li & 3)), pv);
        wave_lds_order();                            // the next tile writes over what others read above
    }
    st.emit(w.massml, w.rows_wg, w.ss, true, w.li, w.lg);
    st.cur_seg = -1;
}

// Values of own tokens `odd` (a bit each) that are not finite, for the rows that see them (zero times one would reach the rows ahead).
template <int DT, int NRB>
__device__ __forceinline__ void add_odd_values(__amdgpu_buffer_rsrc_t values, int pitch, uint32_t odd, int tok0, int lg, Rows<NRB>& st) {
    for (; odd; odd &= odd - 1) {
        const int j = __builtin_ctz(odd);
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            const auto x = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(values, j * pitch + 32 * db + 8 * lg, 0, 0));
            const float v[4] = {Mma<DT>::lo(x.x), Mma<DT>::hi(x.x), Mma<DT>::lo(x.y), Mma<DT>::hi(x.y)};
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (tok0 + j <= st.trow[rb] && !(fabsf(v[r]) < INFINITY)) st.acc[rb][db][r] += v[r];
        }
    }
    st.pin();
}

// A tile of the own block: `ntok` keys (operands as in Parts, from key_at(tb, c)) and staged values; row t sees tokens 0 .. t.  Queries and
// probabilities are two terms of the keys' type: 16 bits each in bf16, whose keys and values have eight.
template <int DT, int NRB, class Key>
__device__ __forceinline__ void own_tile(Rows<NRB>& st, const Parts (&qt)[NRB], Key key_at, const unsigned char* v_read, int tok0, int ntok, const float (&mul)[NRB], int lg) {
    f32x4 sc[NRB][2];
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) sc[rb][0] = sc[rb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            const uint4 kf = key_at(tb, c);
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) {
                sc[rb][tb] = Mma<DT>::run(kf, qt[rb].lo[c], sc[rb][tb]);
                sc[rb][tb] = Mma<DT>::run(kf, qt[rb].hi[c], sc[rb][tb]);
            }
        }
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
        const int last = min(ntok - 1, st.trow[rb] - tok0) - 4 * lg;
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[rb][e >> 2][e & 3] = 16 * (e >> 2) + (e & 3) <= last ? sc[rb][e >> 2][e & 3] : -INFINITY;
    }
    float pv[NRB][8];
    st.template softmax<kOwnLift<DT>>(sc, [&](int rb) { return mul[rb]; }, pv);
    st.template weigh<DT, true>(load_values(v_read), pv);
}

// The run's tiles of the own block, for a wavefront on its own.
template <int DT, int PAIRING, class Table>
__device__ __forceinline__ void own_tiles(const AttnArgs& a, const Table& tbl, const WavePlace& w, const QueryPart& q, float mul, Rows<1>& st) {
    const int lane = 16 * w.lg + w.li, li = w.li, lg = w.lg;
    RunWalk<true> walk(w.t_begin, w.t_end);
    for (;;) {
        const Tile cd = walk.next(tbl, lane);
        if (cd.ntok <= 0) break;
        const int64_t at = ((walk.c_tok + cd.tok0) * a.n_kv_heads + w.hkv) * kD * 2;
        const int pitch = a.n_kv_heads * kD * 2, range = (cd.ntok - 1) * pitch + 2 * kD;
        const auto rk = buffer(a.k_self, at, range), rv = buffer(a.v_self, at, range);
        uint4 kf[2][4], vals[2][4];
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                kf[tb][c] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rk, (16 * tb + li) * pitch + 32 * lg + 128 * (c >> 1) + 16 * (c & 1), 0, 0));
                vals[tb][c] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rv, (16 * tb + li) * pitch + 64 * lg + 16 * c, 0, 0));
            }
        __builtin_amdgcn_sched_barrier(0);
        st.enter(cd.seg, w.massml, w.rows_wg, w.ss, false, li, lg);
        put_angles(a, w.cs, lane, cd.delta, w.my_freq);
        const Parts qt[1] = {to_parts<DT, PAIRING, DT>(q, w.cs, lg)};
        uint32_t odd = 0;                            // tokens with values that are not finite
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            bool any = false;
#pragma unroll
            for (int c = 0; c < 4; ++c) *reinterpret_cast<uint4*>(w.v_lds + (16 * tb + li) * kVRow + 64 * lg + 16 * c) = finite8<DT>(vals[tb][c], any);
            const uint64_t ballot = __ballot(any);
            odd |= (uint32_t)((ballot | ballot >> 16 | ballot >> 32 | ballot >> 48) & 0xffff) << (16 * tb);
        }
        wave_lds_order();
        own_tile<DT, 1>(st, qt, [&](int tb, int c) { return kf[tb][c]; }, w.v_lds + (4 * lg + (li >> 2)) * kVRow + 8 * (li & 3), cd.tok0, cd.ntok, {mul}, lg);
        wave_lds_order();                            // the next tile writes over what others read above
        add_odd_values<DT, 1>(rv, pitch, odd, cd.tok0, lg, st);
    }
}

// Normalised output channels 16 db + 4 lg .. of a lane's row to `out`, or to the split's partial rows.
template <int DT>
__device__ __forceinline__ void store_out(const AttnArgs& a, int64_t q_first, int qrow, int db, int lg, f32x4 o) {
    uint16_t* op = static_cast<uint16_t*>(a.out) + q_first + (int64_t)qrow * kD + 16 * db + 4 * lg;
    *reinterpret_cast<uint2*>(op) = make_uint2(Mma<DT>::pack(o[0], o[1]), Mma<DT>::pack(o[2], o[3]));
}

// ---------------------------------------------------------------------------------------------
// One row block (a decode step: one row per query head of a group): bound by HBM where there are enough tokens.  A wavefront's loads are two
// tiles ahead in registers; a tile's codes meet the query in registers, its values pass through LDS of the wavefront's own.
// Measured: 4 conversations of 24000 to 31000 tokens x 4 heads (60 MB) 19.0 us, in its loop 5.2 TB/s (a 2 GiB copy: 4.9), then 13 000 clocks of
// prologue, merge of the wavefronts and the own tile; one row over 881 tokens x 32 heads 12.1 us (12.6 in a trace), all of it such latency.  (The own tile ahead of
// the loop, under the first tiles' loads: 0.4 us slower.)
// REG_TABLE: the table in every wavefront's registers where it has at most 64 entries (12.1, 20.7 and 18.8 us for the two and 32 conversations of 1000
// to 5000 tokens; from LDS 12.6, 21.8 and 19.5).
template <int DT, int PAIRING, bool REG_TABLE>
__global__ __launch_bounds__(kSoloThreads, 2) void attn_q4_solo_kernel(AttnArgs a, RopeFreq freq, Plan p, Scales s) {
    __shared__ std::conditional_t<REG_TABLE, int, RunTable> lds_tbl;
    __shared__ __attribute__((aligned(16))) unsigned char lds[kSoloWaves * kVTile];
    __shared__ __attribute__((aligned(16))) float2 cs_lds[kSoloWaves][64];
    __shared__ float2 red_ml[kSoloWaves][16];
    static_assert(sizeof(lds) >= kSoloWaves * 8 * kWave * sizeof(f32x4) && sizeof(lds) >= sizeof(SegTable), "the results and the table reuse the V tiles");

    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int li = lane & 15, lg = lane >> 4;
    ask_for_arguments(a, p, s);
    // grid (split, kv head, query)
    const int split = blockIdx.x, hkv = blockIdx.y, b = blockIdx.z;
    const int unit = b * p.units_per_b + hkv;
    const QueryHead qh = load_query_head(a, b, REG_TABLE ? lane : (int)threadIdx.x);
    const int tq = max(min(qh.tq_raw, a.max_tq), 0);
    Rows<1> st;
    st.begin(0, p.group * tq, p.group, a.n_q_heads, hkv, li);
    const int64_t q_first = (int64_t)qh.q0 * a.n_q_heads * kD;
    const QueryPart raw = query_part(a, q_first, st, 0, lg);         // (loads return in order: ahead of the tiles')
    RegSegTable rtbl;
    int total;
    if constexpr (REG_TABLE) {
        rtbl = build_reg_table(a, qh, lane, kTile);
        total = rtbl.total;
    } else {
        build_run_table(a, qh, &lds_tbl, reinterpret_cast<SegTable*>(lds));
        __syncthreads();
        total = lds_tbl.total;
    }
    char* const ws = static_cast<char*>(a.workspace);
    WavePlace w;
    w.li = li; w.lg = lg; w.hkv = hkv; w.rows_wg = p.rows_wg; w.ss = split * kSoloWaves + wave;
    w.t_begin = run_begin(total, p.nsplit * kSoloWaves, w.ss);
    w.t_end = run_begin(total, p.nsplit * kSoloWaves, w.ss + 1);
    w.q_first = q_first;
    w.my_freq = freq.rev[lane];
    w.cs = cs_lds[wave];
    w.v_lds = lds + wave * kVTile;
    w.massml = a.mass ? reinterpret_cast<float2*>(ws + p.off_massml) + (int64_t)unit * p.slots * p.rows_wg : nullptr;
    auto with_table = [&](auto f) __attribute__((always_inline)) {
        if constexpr (REG_TABLE) f(rtbl);
        else f(lds_tbl);
    };

    RunWalk<false> walk(w.t_begin, w.t_end);
    auto fetch = [&](Tile& d, TileRegs& r) __attribute__((always_inline)) {
        with_table([&](const auto& t) { d = walk.next(t, lane); });
        load_tile(a, s, d, walk.c_tok, hkv, li, lg, r);
    };
    Tile d0, d1;
    TileRegs r0, r1;
    fetch(d0, r0);
    fetch(d1, r1);
    const int q_scale = row_scale<DT>(raw);
    const QueryPart q = scaled<DT>(raw, q_scale);
    const float mul = score_unit(a.scale_log2e, q_scale);
    unsigned char* const v_write = w.v_lds + li * kVRow + 64 * lg;
    const unsigned char* const v_read = w.v_lds + (4 * lg + (li >> 2)) * kVRow + 8 * (li & 3);
    Parts qt;
    int q_delta = 0;
    bool have_parts = false, passed_over = false;
    auto step = [&](Tile& d, TileRegs& r) __attribute__((always_inline)) {
        const Tile cd = d;
        // a tile that is passed over counts as one without tokens (no branch around the body: the compiler would keep the accumulators twice)
        const bool take = tile_fits(r, cd.ntok, li, lg);
        const int ntok = take ? cd.ntok : 0;
        passed_over = passed_over || !take;
        st.enter(cd.seg, w.massml, w.rows_wg, w.ss, false, li, lg);
        if (!have_parts || cd.delta != q_delta) {
            have_parts = true;
            q_delta = cd.delta;
            put_angles(a, w.cs, lane, cd.delta, w.my_freq);
            qt = to_parts<DT, PAIRING, CF_F16>(q, w.cs, lg);
        }
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) stage_values(v_write + 16 * tb * kVRow, r.v[tb], take ? scale_of(r.vs[tb]) : 0.f);
        wave_lds_order();
        f32x4 sc[1][2] = {{f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}}};
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) {
                const uint4 kf = key_operand<CF_F16>(r, tb, c, lg);
                sc[0][tb] = Mma<CF_F16>::run(kf, qt.lo[c], sc[0][tb]);
                sc[0][tb] = Mma<CF_F16>::run(kf, qt.hi[c], sc[0][tb]);
            }
        __builtin_amdgcn_sched_barrier(0);
        fetch(d, r);                                 // the registers are free again
        __builtin_amdgcn_sched_barrier(0);
        const Values vf = load_values(v_read);
        __builtin_amdgcn_sched_barrier(0);
        if (ntok < kTile) {                          // (scores of a tile passed over are replaced as well)
            const int lim = ntok - 4 * lg;
#pragma unroll
            for (int e = 0; e < 8; ++e) sc[0][e >> 2][e & 3] = 16 * (e >> 2) + (e & 3) < lim ? sc[0][e >> 2][e & 3] : -INFINITY;
        }
        float pv[1][8];
        st.template softmax<kLift>(sc, [&](int) { return mul; }, pv);
        st.template weigh<CF_F16, false>(vf, pv);
        wave_lds_order();                            // the next step writes over what others read above
    };
    // (left from the middle: with a step skipped the wait for one register set would have to cover the other as well)
    while (d0.ntok > 0) {
        step(d0, r0);
        if (d1.ntok <= 0) break;
        step(d1, r1);
    }
    if (passed_over) {
        if constexpr (DT == CF_BF16) st.lower();
        with_table([&](const auto& t) __attribute__((always_inline)) { odd_tiles<DT, PAIRING, 1>(a, s, t, w, st); });
    }
    with_table([&](const auto& t) __attribute__((always_inline)) {
        if (!holds<true>(t, w.t_begin, w.t_end, lane)) return;
        if (DT == CF_BF16 && !passed_over) st.lower();
        own_tiles<DT, PAIRING>(a, t, w, q, mul, st);
    });
    st.emit(w.massml, w.rows_wg, w.ss, false, li, lg);

    // ---- the wavefronts' results: wavefront w merges channel block w
    st.close();
    if (lg == 0) red_ml[wave][li] = make_float2(st.m_run[0], st.l_run[0]);
    f32x4* const red = reinterpret_cast<f32x4*>(lds);
    __syncthreads();                                 // every wavefront is done with its V tile
#pragma unroll
    for (int db = 0; db < 8; ++db) red[(wave * 8 + db) * kWave + lane] = st.acc[0][db];
    __syncthreads();
    float m = -INFINITY;
#pragma unroll
    for (int x = 0; x < kSoloWaves; ++x) m = fmaxf(m, red_ml[x][li].x);
    const float ms = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < kSoloWaves; ++x) {
        const float2 v = red_ml[x][li];
        const float f = __builtin_amdgcn_exp2f(v.x - ms);
        l += v.y * f;
        o += red[(x * 8 + wave) * kWave + lane] * f;
    }
    o *= l > 0.f ? 1.f / l : l;                      // (a sum that is not a number stays one)
    const int64_t part = (int64_t)unit * p.nsplit + split;
    if (wave == 0 && lg == 0) reinterpret_cast<float2*>(ws + p.off_ml)[part * p.rows_wg + li] = make_float2(m, st.trow[0] >= 0 ? l : 0.f);
    if (p.direct_out) {
        if (st.trow[0] >= 0) store_out<DT>(a, w.q_first, st.qrow[0], wave, lg, o);
    } else {
        *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(ws + p.off_opart) + (part * p.rows_wg + li) * kD + 16 * wave + 4 * lg) = o;
    }
}

// ---------------------------------------------------------------------------------------------
// More row blocks: eight wavefronts share the 32-token tiles that they stage together, two per step, one for each half of the workgroup to stage.
// Bound by the instructions that a SIMD can issue.
//   * HALVES (at most four blocks): a half streams a run of its own, wavefront w of it with block w; the halves meet in LDS at the end.
//   * Otherwise the halves stage every other tile of one run and every wavefront works on both: NB0 blocks in the first half, NB1 in the
//     second (a SIMD has a wavefront of either, so it gets NB0 + NB1).
// A thread loads 8 bytes of a tile's key codes and of its value codes a step ahead of their staging, two ahead of their use, and unpacks them into
// LDS, each once per workgroup, together with a description of the tile and the angles where a segment begins.  One barrier per step.
// Measured: 64 queries of 384 rows x 2 heads over 3000 tokens in 20 segments 179 us (76 GFLOP that the method needs: 425 TFLOP/s; 1.5 times that runs,
// the scores being products of two terms): 6400 clocks per step of two wavefronts, of which the matrix pipe takes 2300 and the vector unit about
// 3000, which add up to most of it; turning the queries is a quarter of the latter.  The halves' staging at opposite ends of a step, or a raised
// priority for the products: no faster.  448 rows x 4 heads over 7500 tokens 35.8 us, 48 rows x 32 heads over 1680 18.7: half of it prologue and tail.
template <int DT, int PAIRING, int NB0, int NB1, bool HALVES>
__global__ __launch_bounds__(kRowsThreads, 2) void attn_q4_rows_kernel(AttnArgs a, RopeFreq freq, Plan p, Scales s) {
    constexpr int kHalfWaves = kRowsWaves / 2, kHalfThreads = kRowsThreads / 2;
    static_assert(!HALVES || (NB0 == 1 && NB1 == 1), "");
    constexpr int kRowsWg = 16 * kHalfWaves * (HALVES ? 1 : NB0 + NB1);
    __shared__ RunTable tbl;
    // tiles of keys and values, the workgroup's queries; after the last tile a V tile per wavefront, then the second half's results
    constexpr int kKeys = 4 * kKTile, kTiles = kKeys + 4 * kVTile, kBytes = kTiles + kRowsWg * kQRow;
    static_assert(kBytes >= kRowsWaves * kVTile && kBytes >= kHalfWaves * 8 * kWave * (int)sizeof(f32x4) && kTiles >= (int)sizeof(SegTable), "");
    __shared__ __attribute__((aligned(16))) unsigned char lds[kBytes];
    __shared__ __attribute__((aligned(16))) float2 cs_lds[kRowsWaves][64];
    __shared__ __attribute__((aligned(16))) int4 desc_lds[2][2];     // tokens, segment, shift and first token of a staged tile
    __shared__ int odd_lds[2][2];                    // step of the last tile there whose scales do not fit fp16; own tiles: tokens with odd values
    __shared__ float2 red_ml[HALVES ? kRowsWg : 1];

    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave), half = wave / kHalfWaves;
    const int li = lane & 15, lg = lane >> 4;
    ask_for_arguments(a, p, s);
    // grid (split, kv head * row groups + row group, query)
    const int split = blockIdx.x, b = blockIdx.z;
    const int hkv = p.n_rg == 1 ? (int)blockIdx.y : (int)div_exact(blockIdx.y, (unsigned)p.n_rg), rg = (int)blockIdx.y - hkv * p.n_rg;
    const int unit = b * p.units_per_b + (int)blockIdx.y;
    const QueryHead qh = load_query_head(a, b, tid);
    const int tq = max(min(qh.tq_raw, a.max_tq), 0);
    const int row0 = rg * kRowsWg;
    const bool wg_rows = row0 < p.group * tq;        // workgroup-uniform
    char* const ws = static_cast<char*>(a.workspace);

    auto body = [&](auto nrb) __attribute__((always_inline)) {
        constexpr int NRB = decltype(nrb)::value;
        // the wavefront's first row, counted from the workgroup's
        const int wrow = HALVES ? 16 * (wave - half * kHalfWaves) : half == 0 ? 16 * NB0 * wave : 16 * (kHalfWaves * NB0 + NB1 * (wave - kHalfWaves));
        Rows<NRB> st;
        st.begin(row0 + wrow, p.group * tq, p.group, a.n_q_heads, hkv, li);
        WavePlace w;
        w.li = li; w.lg = lg; w.hkv = hkv; w.rows_wg = kRowsWg; w.ss = HALVES ? 2 * split + half : split;
        w.q_first = (int64_t)qh.q0 * a.n_q_heads * kD;
        w.my_freq = freq.rev[lane];
        w.cs = cs_lds[wave];
        w.v_lds = lds + wave * kVTile;
        w.massml = a.mass ? reinterpret_cast<float2*>(ws + p.off_massml) + (int64_t)unit * p.slots * kRowsWg + wrow : nullptr;
        if (tid < 4) odd_lds[tid >> 1][tid & 1] = -1;
        unsigned char* const q_lds = lds + kTiles + (wrow + li) * kQRow + 32 * lg;
        QueryPart q[NRB];
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) q[rb] = query_part(a, w.q_first, st, rb, lg);
        __builtin_amdgcn_sched_barrier(0);
        build_run_table(a, qh, &tbl, reinterpret_cast<SegTable*>(lds));
        float mul[NRB];
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            const int scale = row_scale<DT>(q[rb]);
            mul[rb] = score_unit(a.scale_log2e, scale);
            const QueryPart r = scaled<DT>(q[rb], scale);
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(q_lds + rb * 16 * kQRow + 128 * (i >> 1) + 16 * (i & 1)) = r.w[i];
        }
        __syncthreads();
        const int total = wg_rows ? __builtin_amdgcn_readfirstlane(tbl.total) : 0;
        const int runs = HALVES ? 2 * p.nsplit : p.nsplit;
        w.t_begin = run_begin(total, runs, w.ss);
        w.t_end = run_begin(total, runs, w.ss + 1);

        // a half takes the tiles of its own run, or every other one of the workgroup's
        RunWalk<false> walk(w.t_begin, w.t_end);
        if (!HALVES && half == 1) walk.skip(tbl, lane);
        const int row_bytes = (int)(a.store_ts >> 1), scale_bytes = (int)(a.store_ts >> 5);
        const int st_tok = (tid & (kHalfThreads - 1)) >> 3, st_part = tid & 7;       // token and 16 channels that the thread stages
        struct Regs { uint2 k, v; uint32_t ks, vs; };
        auto fetch = [&](Tile& d, Regs& r) __attribute__((always_inline)) {
            d = walk.next(tbl, lane);
            const bool any = d.ntok > 0;
            const int64_t at = any ? (walk.c_tok + d.tok0) * a.store_ts + (int64_t)hkv * a.store_hs : 0;
            if constexpr (!HALVES) walk.skip(tbl, lane);             // (the other half's)
            const int codes = any ? (d.ntok - 1) * row_bytes + kRowBytes : 0, scales = any ? (d.ntok - 1) * scale_bytes + 4 : 0;
            const int off = st_tok * row_bytes + 8 * st_part, soff = st_tok * scale_bytes + (st_part >> 1);
            r.k = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(buffer(a.k_store, at >> 1, codes), off, 0, 0));
            r.v = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(buffer(a.v_store, at >> 1, codes), off, 0, 0));
            r.ks = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(buffer(s.k, at >> 5, scales), soff, 0, 0);
            r.vs = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(buffer(s.v, at >> 5, scales), soff, 0, 0);
        };
        auto angles = [&](int slot, int delta) __attribute__((always_inline)) { cs_lds[slot][lane] = turn_angle(a, delta, w.my_freq); };
        // tile d, loaded to r, to buffer `buf`; the first of a segment or run with its angles, which the half's wavefronts take turns in
        auto stage = [&](const Tile& d, const Regs& r, int buf, int step, bool first) __attribute__((always_inline)) {
            const bool fits = fits_f16(r.ks) && fits_f16(r.vs);
            const float sk = scale_of(r.ks), sv = fits_f16(r.vs) ? scale_of(r.vs) : 0.f;
            unsigned char* const k_to = lds + (2 * buf + half) * kKTile + st_tok * kKRow + 32 * st_part;
            unsigned char* const v_to = lds + kKeys + (2 * buf + half) * kVTile + st_tok * kVRow + 32 * st_part;
            *reinterpret_cast<uint4*>(k_to) = unpack8<CF_F16>(r.k.x, sk);
            *reinterpret_cast<uint4*>(k_to + 16) = unpack8<CF_F16>(r.k.y, sk);
            *reinterpret_cast<uint4*>(v_to) = unpack8<CF_F16>(r.v.x, sv);
            *reinterpret_cast<uint4*>(v_to + 16) = unpack8<CF_F16>(r.v.y, sv);
            if (!fits && st_tok < d.ntok) odd_lds[buf][half] = step;
            if ((tid & (kHalfThreads - 1)) == 0) desc_lds[buf][half] = make_int4(d.ntok, d.seg, d.delta, d.tok0);
            if ((first || d.tok0 == 0) && ((wave ^ step) & (kHalfWaves - 1)) == 0) angles(2 * buf + half, d.delta);
        };
        auto scalar = [](int x) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane(x); };
        Parts qt[NRB];
        auto turn = [&](auto type, int slot) __attribute__((always_inline)) {
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) {
                QueryPart q;
#pragma unroll
                for (int i = 0; i < 4; ++i) q.w[i] = *reinterpret_cast<const uint4*>(q_lds + rb * 16 * kQRow + 128 * (i >> 1) + 16 * (i & 1));
                qt[rb] = to_parts<DT, PAIRING, decltype(type)::value>(q, cs_lds[slot], lg);
            }
        };

        Tile dn;
        Regs r;
        fetch(dn, r);
        stage(dn, r, 0, 0, true);
        fetch(dn, r);
        int q_delta = 0, step = 0;
        bool have_parts = false, passed_over = false;
        const unsigned char* const k_read = lds + li * kKRow + 32 * lg;
        const unsigned char* const v_read = lds + kKeys + (4 * lg + (li >> 2)) * kVRow + 8 * (li & 3);
        for (int buf = 0;; buf ^= 1, ++step) {
            __syncthreads();                         // the step's tiles are staged; every wavefront is done with the other buffer
            const int4 e0 = desc_lds[buf][0], e1 = desc_lds[buf][1];
            const int odd0 = odd_lds[buf][0], odd1 = odd_lds[buf][1];
            if (scalar(e0.x | e1.x) == 0) break;
            stage(dn, r, buf ^ 1, step + 1, false);
            fetch(dn, r);
            const int t_end = HALVES ? half + (scalar(half ? e1.x : e0.x) > 0) : 1 + (scalar(e1.x) > 0);
#pragma unroll 1
            for (int t = HALVES ? half : 0; t < t_end; ++t) {
                const int slot = 2 * buf + t;
                const int all = scalar(t ? e1.x : e0.x), seg = scalar(t ? e1.y : e0.y), delta = scalar(t ? e1.z : e0.z);
                // a tile that is passed over counts as one without tokens (no branch around the body: the compiler would keep the accumulators twice)
                const bool take = scalar(t ? odd1 : odd0) != step;
                const int ntok = take ? all : 0;
                passed_over = passed_over || !take;
                st.enter(seg, w.massml, kRowsWg, w.ss, false, li, lg);
                if (!have_parts || delta != q_delta) {
                    have_parts = true;
                    q_delta = delta;
                    turn(std::integral_constant<int, CF_F16>{}, slot);
                }
                f32x4 sc[NRB][2];
#pragma unroll
                for (int rb = 0; rb < NRB; ++rb) sc[rb][0] = sc[rb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
                // (all of a tile's operands are asked for ahead of the products: else the compiler waits for each)
                uint4 kf[4][2];
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int tb = 0; tb < 2; ++tb)
                        kf[c][tb] = *reinterpret_cast<const uint4*>(k_read + slot * kKTile + 16 * tb * kKRow + 128 * (c >> 1) + 16 * (c & 1));
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                        for (int rb = 0; rb < NRB; ++rb) {
                            sc[rb][tb] = Mma<CF_F16>::run(kf[c][tb], qt[rb].lo[c], sc[rb][tb]);
                            sc[rb][tb] = Mma<CF_F16>::run(kf[c][tb], qt[rb].hi[c], sc[rb][tb]);
                        }
                const Values vf = load_values(v_read + slot * kVTile);
                __builtin_amdgcn_sched_barrier(0);
                if (ntok < kTile) {
                    const int lim = ntok - 4 * lg;
#pragma unroll
                    for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                        for (int e = 0; e < 8; ++e) sc[rb][e >> 2][e & 3] = 16 * (e >> 2) + (e & 3) < lim ? sc[rb][e >> 2][e & 3] : -INFINITY;
                }
                float pv[NRB][8];
                st.template softmax<kLift>(sc, [&](int rb) { return mul[rb]; }, pv);
                st.template weigh<CF_F16, false>(vf, pv);
            }
        }
        const int wg_begin = HALVES ? run_begin(total, runs, 2 * split) : w.t_begin, wg_end = HALVES ? run_begin(total, runs, 2 * split + 2) : w.t_end;
        __syncthreads();                             // every wavefront is done with the tiles and their descriptions
        const bool own_tiles_here = holds<true>(tbl, wg_begin, wg_end, lane);
        if (DT == CF_BF16 && (passed_over || own_tiles_here)) st.lower();
        if (own_tiles_here) {
            // the own block, two tiles of 16-bit keys and values per step
            RunWalk<true> own(w.t_begin, w.t_end);
            if (!HALVES && half == 1) own.skip(tbl, lane);
            const int pitch = a.n_kv_heads * kD * 2;
            have_parts = false;
            for (;;) {
                const Tile d = own.next(tbl, lane);
                const bool any = d.ntok > 0;
                const int64_t at = any ? ((own.c_tok + d.tok0) * a.n_kv_heads + hkv) * kD * 2 : 0;
                if constexpr (!HALVES) own.skip(tbl, lane);
                const int range = any ? (d.ntok - 1) * pitch + 2 * kD : 0;
                const auto rk = buffer(a.k_self, at, range), rv = buffer(a.v_self, at, range);
                const int off = st_tok * pitch + 32 * st_part;
                const uint4 k0 = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rk, off, 0, 0));
                const uint4 k1 = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rk, off + 16, 0, 0));
                const uint4 v0 = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rv, off, 0, 0));
                const uint4 v1 = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rv, off + 16, 0, 0));
                if ((wave & (kHalfWaves - 1)) == 0) angles(half, d.delta);
                if ((tid & (kHalfThreads - 1)) == 0) { desc_lds[0][half] = make_int4(d.ntok, d.seg, d.delta, d.tok0); odd_lds[0][half] = 0; }
                __syncthreads();
                bool not_finite = false;
                unsigned char* const k_to = lds + half * kKTile + st_tok * kKRow + 32 * st_part;
                unsigned char* const v_to = lds + kKeys + half * kVTile + st_tok * kVRow + 32 * st_part;
                reinterpret_cast<uint4*>(k_to)[0] = k0;
                reinterpret_cast<uint4*>(k_to)[1] = k1;
                reinterpret_cast<uint4*>(v_to)[0] = finite8<DT>(v0, not_finite);
                reinterpret_cast<uint4*>(v_to)[1] = finite8<DT>(v1, not_finite);
                if (not_finite) atomicOr(&odd_lds[0][half], 1 << st_tok);
                __syncthreads();
                const int4 e0 = desc_lds[0][0], e1 = desc_lds[0][1];
                if (scalar(e0.x | e1.x) == 0) break;
                const int t_end = HALVES ? half + (scalar(half ? e1.x : e0.x) > 0) : 1 + (scalar(e1.x) > 0);
#pragma unroll 1
                for (int t = HALVES ? half : 0; t < t_end; ++t) {
                    const int ntok = scalar(t ? e1.x : e0.x), seg = scalar(t ? e1.y : e0.y), delta = scalar(t ? e1.z : e0.z), tok0 = scalar(t ? e1.w : e0.w);
                    st.enter(seg, w.massml, kRowsWg, w.ss, false, li, lg);
                    if (!have_parts || delta != q_delta) {
                        have_parts = true;
                        q_delta = delta;
                        turn(std::integral_constant<int, DT>{}, t);
                    }
                    own_tile<DT, NRB>(st, qt, [&](int tb, int c) {
                        return *reinterpret_cast<const uint4*>(k_read + t * kKTile + 16 * tb * kKRow + 128 * (c >> 1) + 16 * (c & 1));
                    }, v_read + t * kVTile, tok0, ntok, mul, lg);
                    const uint32_t odd = (uint32_t)scalar(odd_lds[0][t]);
                    if (odd) {
                        const int64_t tok = scalar64(tbl.tok[seg]) + tok0;
                        add_odd_values<DT, NRB>(buffer(a.v_self, (tok * a.n_kv_heads + hkv) * kD * 2, (ntok - 1) * pitch + 2 * kD), pitch, odd, tok0, lg, st);
                    }
                }
                __syncthreads();                     // every wavefront is done with the tiles and their descriptions
            }
            __syncthreads();
        }
        if (passed_over) odd_tiles<DT, PAIRING, NRB>(a, s, tbl, w, st);
        st.emit(w.massml, kRowsWg, w.ss, false, li, lg);
        st.close();
        if constexpr (HALVES) {                      // the second half's rows join the first's
            f32x4* const red = reinterpret_cast<f32x4*>(lds) + (wave - half * kHalfWaves) * 8 * kWave + lane;
            __syncthreads();
            if (half == 1) {
                if (lg == 0) red_ml[wrow + li] = make_float2(st.m_run[0], st.l_run[0]);
#pragma unroll
                for (int db = 0; db < 8; ++db) red[db * kWave] = st.acc[0][db];
            }
            __syncthreads();
            if (half == 1) return;
            const float2 o = red_ml[wrow + li];
            const float m = fmaxf(st.m_run[0], o.x), ms = m == -INFINITY ? 0.f : m;
            const float f = __builtin_amdgcn_exp2f(st.m_run[0] - ms), g = __builtin_amdgcn_exp2f(o.x - ms);
            st.m_run[0] = m;
            st.l_run[0] = st.l_run[0] * f + o.y * g;
#pragma unroll
            for (int db = 0; db < 8; ++db) st.acc[0][db] = st.acc[0][db] * f + red[db * kWave] * g;
        }
        const int64_t part = (int64_t)unit * p.nsplit + split;
        float2* const ml = reinterpret_cast<float2*>(ws + p.off_ml) + part * kRowsWg + wrow;
        float* const opart = reinterpret_cast<float*>(ws + p.off_opart) + (part * kRowsWg + wrow) * kD;
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            const float l = st.l_run[rb], inv = l > 0.f ? 1.f / l : l;       // (a sum that is not a number stays one)
            if (lg == 0) ml[16 * rb + li] = make_float2(st.m_run[rb], st.trow[rb] >= 0 ? l : 0.f);
            if (st.trow[rb] < 0) continue;
#pragma unroll
            for (int db = 0; db < 8; ++db) {
                if (p.direct_out) store_out<DT>(a, w.q_first, st.qrow[rb], db, lg, st.acc[rb][db] * inv);
                else *reinterpret_cast<f32x4*>(opart + (16 * rb + li) * kD + 16 * db + 4 * lg) = st.acc[rb][db] * inv;
            }
        }
    };
    if constexpr (NB0 == NB1) {
        body(std::integral_constant<int, NB0>{});
    } else {                                         // (both bodies pass the same barriers: the steps are the workgroup's)
        if (half == 0) body(std::integral_constant<int, NB0>{});
        else body(std::integral_constant<int, NB1>{});
    }
}

// ---------------------------------------------------------------------------------------------
// What follows the attention: workgroups that work out masses (of one table entry each) and workgroups that merge the splits' partial rows, in one
// launch, since they do not depend on each other.  Both are bound by latency.

// Merges a row's partial rows, a wavefront per row: lane s holds the statistics of split s, then a lane two channels.
template <int DT>
__device__ __forceinline__ void merge_row(const AttnArgs& a, const Plan& p, int b, int unit_of_b, int row, int lane) {
    const int unit = b * p.units_per_b + unit_of_b;
    const int hkv = p.n_rg == 1 ? unit_of_b : (int)div_exact((unsigned)unit_of_b, (unsigned)p.n_rg), rg = unit_of_b - hkv * p.n_rg;
    const char* ws = static_cast<const char*>(a.workspace);
    const int64_t first = (int64_t)unit * p.nsplit * p.rows_wg + row;
    const float2* const ml = reinterpret_cast<const float2*>(ws + p.off_ml) + first;
    const float2* const opart = reinterpret_cast<const float2*>(ws + p.off_opart) + first * (kD / 2) + lane;
    const int q0 = a.q_off[b], q1 = a.q_off[b + 1];
    constexpr int kBatch = 8;
    // everything is requested before anything is waited for; loads past the splits read the last one again
    const float2 stat = ml[(int64_t)min(lane, p.nsplit - 1) * p.rows_wg];
    float2 v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) v[i] = opart[(int64_t)min(i, p.nsplit - 1) * p.rows_wg * (kD / 2)];
    const int tq = max(min(q1 - q0, a.max_tq), 0);
    const int m2 = rg * p.rows_wg + row;
    if (m2 >= p.group * tq) return;
    const float mx = wave_max(lane < p.nsplit ? stat.x : -INFINITY);
    const float m = mx == -INFINITY ? 0.f : mx;
    const float weight = lane < p.nsplit ? stat.y * __builtin_amdgcn_exp2f(stat.x - m) : 0.f;
    const float l = wave_sum_dpp(weight);
    float2 o = make_float2(0.f, 0.f);
    for (int s0 = 0; s0 < p.nsplit; s0 += kBatch) {
        float2 x[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) x[i] = v[i];
        if (s0 + kBatch < p.nsplit) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i) v[i] = opart[(int64_t)min(s0 + kBatch + i, p.nsplit - 1) * p.rows_wg * (kD / 2)];
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (s0 + i >= p.nsplit) break;
            const float f = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, weight), s0 + i));
            o.x += x[i].x * f;
            o.y += x[i].y * f;
        }
    }
    const float inv = l > 0.f ? 1.f / l : l;
    const int t = (int)div_exact((unsigned)m2, (unsigned)p.group), g = m2 - t * p.group;
    uint32_t* op = static_cast<uint32_t*>(a.out) + (((int64_t)q0 + t) * a.n_q_heads + hkv * p.group + g) * (kD / 2) + lane;
    *op = Mma<DT>::pack(o.x * inv, o.y * inv);
}

// Per-segment attention mass: over the units, the runs that hold the segment's tiles and the rows, sum * exp2(reference - row maximum) / row sum, in
// a fixed order.  Then S += mass (Alg. 2): a document slot's first entry works out the masses of all of the slot's entries and adds them up in table
// order.
__device__ __forceinline__ void entry_mass(const AttnArgs& a, const Plan& p, int b, int entry) {
    __shared__ SegTable tbl;
    __shared__ float part_sum[kMergeThreads / kWave];
    __shared__ float2 stat[kMassRows];               // of the units at hand: row maximum, 1 / row sum
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const bool in_regs = a.seg_stride <= kWave;      // every wavefront keeps the table in registers
    const QueryHead qh = load_query_head(a, b, in_regs ? lane : tid);
    RegSegTable reg;
    if (in_regs) reg = build_reg_table(a, qh, lane, kTile);
    else build_table(a, qh, &tbl, kTile);
    const int n = in_regs ? reg.n : tbl.n, total = in_regs ? reg.total : tbl.tile0[tbl.n];
    if (entry >= n) return;
    auto doc_of = [&](int s) { return in_regs ? __builtin_amdgcn_readlane(qh.seg.doc, s) : tbl.doc[s]; };
    const char* ws = static_cast<const char*>(a.workspace);
    const int tq = max(min(qh.tq_raw, a.max_tq), 0), n_rows = p.group * tq;
    const int nsub = p.nsplit * p.runs;
    const int log_rows = p.rows_wg <= 16 ? 4 : p.rows_wg <= 64 ? 6 : p.rows_wg <= 128 ? 7 : 8, rows = 1 << log_rows;
    const int row = tid & (rows - 1), first = tid >> log_rows, per = (int)blockDim.x >> log_rows;
    const int chunk = kMassRows >> log_rows;         // units at a time
    const float inv_rg = 1.f / (float)p.n_rg, inv_nsub = 1.f / (float)nsub;
    // whether `row` of unit u (of the query) is one of the query's (fewer than 2^21 units)
    auto is_row = [&](int u) {
        const int rg = p.n_rg == 1 ? 0 : u - (int)div_small((unsigned)u, (unsigned)p.n_rg, inv_rg) * p.n_rg;
        return row < p.rows_wg && rg * p.rows_wg + row < n_rows;
    };
    constexpr int kBatch = 8;                        // loads in flight
    auto mass_of = [&](int s) {
        const int ts = in_regs ? __builtin_amdgcn_readlane(reg.t0, s) : tbl.tile0[s], te = in_regs ? __builtin_amdgcn_readlane(reg.t1, s) : tbl.tile0[s + 1];
        float sum = 0.f;
        if (te > ts) {
            const int sub0 = run_of(total, nsub, ts), sub1 = run_of(total, nsub, te - 1), n_sub = sub1 - sub0 + 1;
            const float inv_sub = 1.f / (float)n_sub;
            const int du = (int)div_small((unsigned)per, (unsigned)n_sub, inv_sub), ds = per - du * n_sub;
            const int u_first = (int)div_small((unsigned)first, (unsigned)n_sub, inv_sub);
            for (int u0 = 0; u0 < p.units_per_b; u0 += chunk) {
                const int nu = min(chunk, p.units_per_b - u0);
                const int64_t unit0 = (int64_t)b * p.units_per_b + u0;
                const float2* const ml = reinterpret_cast<const float2*>(ws + p.off_ml) + unit0 * p.nsplit * p.rows_wg + row;
                __syncthreads();                     // stat is free
                for (int u = first; u < nu; u += per) {
                    float m = -INFINITY, l = 0.f;
                    if (!is_row(u0 + u)) {
                    } else if (p.nsplit == 1) {
                        const float2 v = ml[(int64_t)u * p.rows_wg];
                        m = v.x;
                        l = v.y;
                    } else {
                        for (int s0 = 0; s0 < p.nsplit; s0 += kBatch) {
                            float2 v[kBatch];
                            float top = m;
#pragma unroll
                            for (int j = 0; j < kBatch; ++j) v[j] = ml[((int64_t)u * p.nsplit + min(s0 + j, p.nsplit - 1)) * p.rows_wg];
#pragma unroll
                            for (int j = 0; j < kBatch; ++j) top = fmaxf(top, v[j].x);
                            const float safe = top == -INFINITY ? 0.f : top;
                            l *= __builtin_amdgcn_exp2f(m - safe);
#pragma unroll
                            for (int j = 0; j < kBatch; ++j)
                                if (s0 + j < p.nsplit) l += v[j].y * __builtin_amdgcn_exp2f(v[j].x - safe);
                            m = top;
                        }
                    }
                    stat[(u << log_rows) + row] = make_float2(m == -INFINITY ? 0.f : m, l > 0.f ? 1.f / l : l);
                }
                __syncthreads();
                // items: unit and run, item first + k * per stepped without a division; a group's threads take an item's rows side by side
                const float2* const pairs = reinterpret_cast<const float2*>(ws + p.off_massml) + (unit0 * p.slots + s + sub0) * p.rows_wg + row;
                int u = u_first, sub = first - u_first * n_sub;
                for (int left = nu * n_sub - first; left > 0; left -= kBatch * per) {
                    float2 v[kBatch], r[kBatch];
#pragma unroll
                    for (int j = 0; j < kBatch; ++j) {
                        bool take = j * per < left && is_row(u0 + u);
                        // a run between a segment's first and last may own no tile at all: its slot was not written
                        if (total < nsub) {
                            const unsigned at = (unsigned)(total * (sub0 + sub));
                            take = take && div_small(at, (unsigned)nsub, inv_nsub) < div_small(at + (unsigned)total, (unsigned)nsub, inv_nsub);
                        }
                        v[j] = r[j] = make_float2(0.f, 0.f);
                        if (take) {
                            v[j] = pairs[((int64_t)u * p.slots + sub) * p.rows_wg];
                            r[j] = stat[(u << log_rows) + row];
                        }
                        u += du;
                        sub += ds;
                        if (sub >= n_sub) { sub -= n_sub; ++u; }
                    }
#pragma unroll
                    for (int j = 0; j < kBatch; ++j) sum += v[j].y * __builtin_amdgcn_exp2f(v[j].x - r[j].x) * r[j].y;
                }
            }
        }
        sum = wave_sum_dpp(sum);
        __syncthreads();
        if (lane == 0) part_sum[tid / kWave] = sum;
        __syncthreads();
        float all = part_sum[0];
#pragma unroll
        for (int w = 1; w < kMergeThreads / kWave; ++w)
            if (w * kWave < (int)blockDim.x) all += part_sum[w];
        return all;
    };
    const float mine = mass_of(entry);
    if (tid == 0) a.mass[(int64_t)b * a.seg_stride + entry] = mine;
    if (a.score_accum == nullptr) return;
    const int d = doc_of(entry);
    if (d < 0 || d >= a.score_stride) return;
    float sum = mine;
    for (int j = 0; j < n; ++j) {                    // workgroup-uniform
        if (doc_of(j) != d) continue;
        if (j < entry) return;
        if (j > entry) sum += mass_of(j);
    }
    if (tid == 0) a.score_accum[(int64_t)b * a.score_stride + d] += sum;
}

template <int DT>
__global__ __launch_bounds__(kMergeThreads) void q4_merge_kernel(AttnArgs a, Plan p) {
    // grid (table entries, then rows of all units; query)
    const int b = blockIdx.y, entries = a.mass != nullptr ? a.seg_stride : 0;
    if ((int)blockIdx.x < entries) {
        entry_mass(a, p, b, blockIdx.x);
        return;
    }
    const int row = __builtin_amdgcn_readfirstlane(((int)blockIdx.x - entries) * ((int)blockDim.x / kWave) + (int)threadIdx.x / kWave);
    const int unit = (int)div_exact((unsigned)row, (unsigned)p.rows_wg);
    if (unit < p.units_per_b) merge_row<DT>(a, p, b, unit, row - unit * p.rows_wg, threadIdx.x & (kWave - 1));
}

}  // namespace
}  // namespace q4

size_t q4_workspace_bytes(const cf_layer_desc* d, int32_t batch, int32_t max_tq, int32_t seg_stride, int64_t max_kv_tokens) {
    return q4::make_plan(d->n_q_heads, d->n_kv_heads, batch, max_tq, seg_stride, max_kv_tokens).total;
}

cf_status launch_attention_q4(const AttnArgs& a, const q4::Scales& sc, const RopeFreq& f, hipStream_t s) {
    using namespace q4;
    const Plan p = make_plan(a.n_q_heads, a.n_kv_heads, a.batch, a.max_tq, a.seg_stride, a.max_kv_tokens);
    if (a.batch > 65535 || p.units_per_b > 65535 || p.units == INT32_MAX) {
        set_error("neither batch nor n_kv_heads * row groups may exceed 65535 on this path, nor both together 2^31 workgroups");
        return CF_ERR_UNSUPPORTED;
    }
    const dim3 grid((unsigned)p.nsplit, (unsigned)p.units_per_b, (unsigned)a.batch);
    auto go = [&](auto dt, auto pairing) {
        constexpr int DT = decltype(dt)::value, PAIRING = decltype(pairing)::value;
        if (p.solo) {
            if (a.seg_stride <= kWave) hipLaunchKernelGGL((attn_q4_solo_kernel<DT, PAIRING, true>), grid, dim3(kSoloThreads), 0, s, a, f, p, sc);
            else hipLaunchKernelGGL((attn_q4_solo_kernel<DT, PAIRING, false>), grid, dim3(kSoloThreads), 0, s, a, f, p, sc);
        } else if (p.halves) {
            hipLaunchKernelGGL((attn_q4_rows_kernel<DT, PAIRING, 1, 1, true>), grid, dim3(kRowsThreads), 0, s, a, f, p, sc);
        } else if (p.rows_wg == 128) {
            hipLaunchKernelGGL((attn_q4_rows_kernel<DT, PAIRING, 1, 1, false>), grid, dim3(kRowsThreads), 0, s, a, f, p, sc);
        } else if (p.rows_wg == 192) {
            hipLaunchKernelGGL((attn_q4_rows_kernel<DT, PAIRING, 2, 1, false>), grid, dim3(kRowsThreads), 0, s, a, f, p, sc);
        } else {
            hipLaunchKernelGGL((attn_q4_rows_kernel<DT, PAIRING, 2, 2, false>), grid, dim3(kRowsThreads), 0, s, a, f, p, sc);
        }
    };
    auto by_pairing = [&](auto dt) {
        if (a.pairing == CF_ROPE_HALF) go(dt, std::integral_constant<int, CF_ROPE_HALF>{});
        else go(dt, std::integral_constant<int, CF_ROPE_INTERLEAVED>{});
    };
    const bool bf16 = a.dtype == CF_BF16;
    if (bf16) by_pairing(std::integral_constant<int, CF_BF16>{});
    else by_pairing(std::integral_constant<int, CF_F16>{});
    CF_HIP(hipGetLastError());
    const int64_t rows = p.direct_out ? 0 : (int64_t)p.units_per_b * p.rows_wg, per = p.merge_threads / kWave;
    const int64_t blocks = (a.mass != nullptr ? a.seg_stride : 0) + (rows + per - 1) / per;
    if (blocks > 0) {
        const dim3 after((unsigned)blocks, (unsigned)a.batch);
        if (bf16) hipLaunchKernelGGL(q4_merge_kernel<CF_BF16>, after, dim3((unsigned)p.merge_threads), 0, s, a, p);
        else hipLaunchKernelGGL(q4_merge_kernel<CF_F16>, after, dim3((unsigned)p.merge_threads), 0, s, a, p);
        CF_HIP(hipGetLastError());
    }
    return CF_OK;
}

}  // namespace cf
