// Prefill and decode attention over a cache store in 4 bits for gfx950 (head_dim 128, 16-bit queries and outputs).
//
// A stored key or value row is 128 codes of four bits and four scale bytes (32 channels each).  What is moved to other positions is the query
// and not the keys: (R_delta k) . q = k . (R_-delta q), once per segment instead of once per key (Eq. 5), and the keys stay exact.
// Scores.  The turned query, scaled by a power of two of its row, enters as two parts: its fp16 value, multiplied with the keys unpacked to fp16
// (exact: at most two significant bits and an exponent inside fp16's) by v_mfma_f32_16x16x32_f16, and the remainder in e4m3, multiplied with
// the codes and scale bytes as they lie in memory by v_mfma_scale_f32_16x16x128_f8f6f4: 15 bits of the query in all.  (That instruction alone, with
// three e4m3 terms, costs the same matrix cycles and no unpacking, but sums its 128 products with an error of up to 2^-13 of the
// largest one: attention masses were off by 2e-6 to 5e-6, by ... with the main part in fp16.)
// Values are unpacked to fp16, staged in LDS and read transposed; probabilities are rounded to fp16 (2^-11), sums, maxima and accumulators
// are fp32.  Tiles with a scale outside fp16's exponents are left to a second pass over the run in which keys meet a query of three e4m3 terms
// and values and probabilities are bf16, the latter as value and remainder.
//
// Work: the rows that share a kv head (row m = t * group + head) are cut into 16-row blocks.
//   * One block (decode steps): attn_q4_solo_kernel, each of eight wavefronts streams a run of 32-token tiles of its own; they meet in LDS at the end.
//   * More: attn_q4_rows_kernel, four wavefronts own one or two blocks each and share the tiles that they stage together.
// Splits (workgroups of the same rows) leave fp32 partial rows that q4_combine_kernel merges; q4_mass_kernel reduces the (reference, sum) pairs
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

constexpr int kSoloThreads = kSoloWaves * kWave, kRowsThreads = kRowsWaves * kWave;
constexpr int kVRow = 288;                           // bytes per token of a staged V tile
constexpr int kVTile = kTile * kVRow;
constexpr int kRowBytes = 64;                        // codes of a row
constexpr int kQRow = 272;                           // bytes per row of queries in LDS
constexpr float kProbLimit = attn::kProbLimit;

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

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

// Walks the tiles of a run that lie in the store, or (OWN) in the own block.
template <bool OWN>
struct RunWalk {
    int next_tile, t_end;
    int c_seg = -1, c_first = 0, c_end = 0, c_vis = 0, c_delta = 0;
    int64_t c_tok = 0;          // first token of the cached segment in its tensor
    bool others = false;        // tiles of the other kind were passed over

    __device__ __forceinline__ RunWalk(int begin, int end) : next_tile(begin), t_end(end) {}

    // The next tile, or one with ntok == 0 when none is left.
    template <class Table>
    __device__ __forceinline__ Tile next(const Table& tbl, int lane) {
        Tile d;
        d.seg = 0; d.tok0 = 0; d.ntok = 0; d.delta = 0; d.self = 0;
        while (next_tile < t_end) {
            if (next_tile >= c_end) {
                const attn::FoundSegment f = attn::find_segment(tbl, next_tile, lane, c_seg);
                c_seg = f.seg;
                c_first = f.first;
                c_end = f.end;
                c_vis = f.vis;
                c_delta = f.delta;
                c_tok = f.tok;
                if ((f.self != 0) != OWN) {
                    others = true;
                    next_tile = f.end;
                    continue;
                }
            }
            d.seg = c_seg;
            d.tok0 = (next_tile - c_first) * kTile;
            d.ntok = max(0, min(kTile, c_vis - d.tok0));
            d.delta = c_delta;
            ++next_tile;
            break;
        }
        return d;
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
// The exponent byte of the power of two that queries are scaled down by: the largest channel, turned by any angle, comes to at most 2^7 * sqrt(2).
template <int DT>
__device__ __forceinline__ int scale_byte_of(uint32_t top) { return max((int)(__float_as_uint(Mma<DT>::lo(top)) >> 23) - 6, 27); }
template <int DT>
__device__ __forceinline__ int row_scale(const QueryPart& q) {
    uint32_t top = largest<DT>(q);
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    return scale_byte_of<DT>(top);
}

__device__ __forceinline__ float scale_down(int scale) { return __uint_as_float((uint32_t)(254 - scale) << 23); }

// A 16-row block of turned queries: fp16 values (hi[s]: channels 32 lg + 8 s .. + 7) and what is left, 2^11 times larger, in e4m3.
constexpr int kLoScale = 127 - 11;
struct Parts { uint4 hi[4]; i32x8 lo; };

// `down`: scales the queries, if `cs` does not.
template <int DT, int PAIRING>
__device__ __forceinline__ Parts to_parts(const QueryPart& q, float down, const float2* cs, int lg) {
    Parts r;
    uint32_t h[2][8];                                // fp16 pairs of either half
    auto split = [&](float (&v)[4], int w, uint32_t (&h)[8], int at) __attribute__((always_inline)) {
        h[at] = Mma<CF_F16>::pack(v[0] * down, v[1] * down);
        h[at + 1] = Mma<CF_F16>::pack(v[2] * down, v[3] * down);
        auto rest = [&](int i, float x) { return fmaf(v[i], down, -x) * 2048.f; };       // exact
        const int packed = __builtin_amdgcn_cvt_pk_fp8_f32(rest(0, Mma<CF_F16>::lo(h[at])), rest(1, Mma<CF_F16>::hi(h[at])), 0, false);
        r.lo[w] = __builtin_amdgcn_cvt_pk_fp8_f32(rest(2, Mma<CF_F16>::lo(h[at + 1])), rest(3, Mma<CF_F16>::hi(h[at + 1])), packed, true);
    };
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        float a[4], b[4];
        turn4<DT, PAIRING>(q, n, cs, lg, a, b);
        split(a, n, h[0], 2 * n);
        split(b, 4 + n, h[1], 2 * n);
        __builtin_amdgcn_sched_barrier(0);           // few floats at a time
    }
    // A lane has turned channels 16 lg .. and 64 + 16 lg .. (both of a slice), the fp16 fragments want 32 lg ...: lane groups 0 | 1 | 2 | 3 take the
    // first halves of groups 0, 1 | 2, 3 and the second halves of 0, 1 | 2, 3
    uint32_t f[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const auto x = __builtin_amdgcn_permlane32_swap(h[0][i], h[1][i], false, false);
        const auto y = __builtin_amdgcn_permlane16_swap(x[0], x[1], false, false);
        f[i] = y[0];
        f[8 + i] = y[1];
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) r.hi[s] = make_uint4(f[4 * s], f[4 * s + 1], f[4 * s + 2], f[4 * s + 3]);
    return r;
}

// The same as three terms of e4m3, 16 times larger from one to the next, for keys of any scale.
constexpr int kTerms = 3;
struct Terms { i32x8 t[kTerms]; };

template <int DT, int PAIRING>
__device__ __forceinline__ Terms to_terms(const QueryPart& q, int scale, const float2* cs, int lg) {
    const float down = scale_down(scale);
    Terms r;
    auto split = [&](float (&v)[4], int w) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= down;
#pragma unroll
        for (int k = 0; k < kTerms; ++k) {
            int packed = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
            packed = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], packed, true);
            r.t[k][w] = packed;
            if (k + 1 < kTerms) {                    // what is left: exact
                const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(packed, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(packed, true);
                v[0] = (v[0] - lo[0]) * 16.f;
                v[1] = (v[1] - lo[1]) * 16.f;
                v[2] = (v[2] - hi[0]) * 16.f;
                v[3] = (v[3] - hi[1]) * 16.f;
            }
        }
    };
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        float a[4], b[4];
        turn4<DT, PAIRING>(q, n, cs, lg, a, b);
        split(a, n);
        split(b, 4 + n);
        __builtin_amdgcn_sched_barrier(0);
    }
    return r;
}

__device__ __forceinline__ f32x4 mma_fp4(i32x4 k, int k_scale, const i32x8& q, int q_scale, f32x4 c) {
    const i32x8 a = {k[0], k[1], k[2], k[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q, c, 4, 0, 0, k_scale, 0, q_scale);
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

// two floats as 16-bit values and what is left of them
template <int DT>
__device__ __forceinline__ void split2(float x, float y, uint32_t& hi, uint32_t& lo) {
    hi = Mma<DT>::pack(x, y);
    lo = Mma<DT>::pack(x - Mma<DT>::lo(hi), y - Mma<DT>::hi(hi));
}
template <int DT>
__device__ __forceinline__ void split8(const float (&v)[8], uint4& hi, uint4& lo) {
    split2<DT>(v[0], v[1], hi.x, lo.x);
    split2<DT>(v[2], v[3], hi.y, lo.y);
    split2<DT>(v[4], v[5], hi.z, lo.z);
    split2<DT>(v[6], v[7], hi.w, lo.w);
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
    // Online softmax (exp2 domain) of scores sc, in units of mul(block), against a stale row maximum: probabilities pv; see kProbLimit.
    template <class F>
    __device__ __forceinline__ void softmax(f32x4 (&sc)[NRB][2], F mul, float (&pv)[NRB][8]) {
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
            off = off || !(lsum[rb] <= kProbLimit) || m_run[rb] == -INFINITY;
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
    // O^T += V^T P^T, V staged in the type VT.  EXACT: P as value and remainder.
    template <int VT, bool EXACT>
    __device__ __forceinline__ void weigh(const unsigned char* v_read, const float (&pv)[NRB][8]) {
        uint4 ph[NRB], pl[NRB];
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) split8<VT>(pv[rb], ph[rb], pl[rb]);
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)(v_read + 32 * db));
            const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)(v_read + 32 * db + 16 * kVRow));
            const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
            const uint4 va = make_uint4(l2.x, l2.y, h2.x, h2.y);
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) {
                if constexpr (EXACT) acc[rb][db] = Mma<VT>::run(va, pl[rb], acc[rb][db]);
                acc[rb][db] = Mma<VT>::run(va, ph[rb], acc[rb][db]);
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

// A tile of the store for a wavefront on its own: token 16 tb + li, 32 channels from 32 lg on.
struct TileRegs { i32x4 k[2], v[2]; uint32_t ks[2], vs[2]; };
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
        const int off = (16 * tb + li) * row_bytes + 16 * lg, soff = (16 * tb + li) * scale_bytes + lg;
        r.k[tb] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, off, 0, 0));
        r.v[tb] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, off, 0, 0));
        r.ks[tb] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(sk, soff, 0, 0);
        r.vs[tb] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(sv, soff, 0, 0);
    }
}
__device__ __forceinline__ bool tile_fits(const TileRegs& r, int ntok, int li) {
    return __all(((fits_f16(r.ks[0]) && fits_f16(r.vs[0])) || li >= ntok) && ((fits_f16(r.ks[1]) && fits_f16(r.vs[1])) || 16 + li >= ntok));
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

// cos and sin of delta's 64 angles to LDS, times `down`
__device__ __forceinline__ void put_angles(float2* cs, int lane, int delta, double my_freq, float down) {
    wave_lds_order();
    const float2 c = rope_cos_sin_fast(delta, my_freq);
    cs[lane] = make_float2(c.x * down, c.y * down);
    wave_lds_order();
}

template <int NRB>
__device__ __forceinline__ QueryPart query_part(const AttnArgs& a, const WavePlace& w, const Rows<NRB>& st, int rb) {
    int row = st.qrow[rb];
    asm volatile("" : "+v"(row));                    // its addresses are worked out anew, not kept through the loops
    return load_query(static_cast<const uint16_t*>(a.q) + w.q_first + (int64_t)row * kD, st.trow[rb] >= 0, w.lg);
}

// The second pass over a run: the tiles whose scales do not fit fp16, with keys as codes, the query in three e4m3 terms and values and
// probabilities in bf16, the latter as value and remainder.  The segments' slots hold sums already.
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
        if (tile_fits(r, d.ntok, w.li)) continue;
        st.enter(d.seg, w.massml, w.rows_wg, w.ss, true, w.li, w.lg);
        put_angles(w.cs, lane, d.delta, w.my_freq, 1.f);
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                *reinterpret_cast<uint4*>(w.v_lds + (16 * tb + w.li) * kVRow + 64 * w.lg + 16 * c) = unpack8<CF_BF16>(r.v[tb][c], scale_of(r.vs[tb]));
        wave_lds_order();
        f32x4 sc[NRB][2];
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            const QueryPart q = query_part(a, w, st, rb);
            const int scale = row_scale<DT>(q);
            const Terms qt = to_terms<DT, PAIRING>(q, scale, w.cs, w.lg);
            sc[rb][0] = sc[rb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = kTerms - 1; k >= 0; --k)    // the smallest terms first
#pragma unroll
                for (int tb = 0; tb < 2; ++tb) sc[rb][tb] = mma_fp4(r.k[tb], (int)r.ks[tb], qt.t[k], scale - 4 * k, sc[rb][tb]);
            const int lim = d.ntok - 4 * w.lg;
#pragma unroll
            for (int e = 0; e < 8; ++e) sc[rb][e >> 2][e & 3] = 16 * (e >> 2) + (e & 3) < lim ? sc[rb][e >> 2][e & 3] : -INFINITY;
        }
        float pv[NRB][8];
        st.softmax(sc, [&](int) { return a.scale_log2e; }, pv);
        st.template weigh<CF_BF16, true>(w.v_lds + (4 * w.lg + (w.li >> 2)) * kVRow + 8 * (w.li & 3), pv);
        wave_lds_order();                            // the next tile writes over what others read above
    }
    st.emit(w.massml, w.rows_wg, w.ss, true, w.li, w.lg);
    st.cur_seg = -1;
}

// The run's tiles of the own block: 16-bit keys and values, queries and probabilities as value and remainder; row t sees tokens 0 .. t.
template <int DT, int PAIRING, int NRB, class Table>
__device__ __forceinline__ void own_tiles(const AttnArgs& a, const Table& tbl, const WavePlace& w, Rows<NRB>& st) {
    const int lane = 16 * w.lg + w.li, li = w.li, lg = w.lg;
    RunWalk<true> walk(w.t_begin, w.t_end);
    for (;;) {
        const Tile cd = walk.next(tbl, lane);
        if (cd.ntok <= 0) break;
        st.enter(cd.seg, w.massml, w.rows_wg, w.ss, false, li, lg);
        put_angles(w.cs, lane, cd.delta, w.my_freq, 1.f);
        const int64_t at = ((walk.c_tok + cd.tok0) * a.n_kv_heads + w.hkv) * kD * 2;
        const int pitch = a.n_kv_heads * kD * 2, range = (cd.ntok - 1) * pitch + 2 * kD;
        const auto rk = buffer(a.k_self, at, range), rv = buffer(a.v_self, at, range);
        uint4 kf[2][4];
        uint32_t odd = 0;                            // tokens with values that are not finite
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            bool any = false;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                kf[tb][c] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rk, (16 * tb + li) * pitch + 32 * lg + 128 * (c >> 1) + 16 * (c & 1), 0, 0));
                const uint4 v = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rv, (16 * tb + li) * pitch + 64 * lg + 16 * c, 0, 0));
                *reinterpret_cast<uint4*>(w.v_lds + (16 * tb + li) * kVRow + 64 * lg + 16 * c) = finite8<DT>(v, any);
            }
            const uint64_t ballot = __ballot(any);
            odd |= (uint32_t)((ballot | ballot >> 16 | ballot >> 32 | ballot >> 48) & 0xffff) << (16 * tb);
        }
        wave_lds_order();
        f32x4 sc[NRB][2];
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            const QueryPart q = query_part(a, w, st, rb);
            sc[rb][0] = sc[rb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 2; ++c) {            // channels 8c .. 8c + 7 of either half
                float a0[4], b0[4], a1[4], b1[4];
                turn4<DT, PAIRING>(q, 2 * c, w.cs, lg, a0, b0);
                turn4<DT, PAIRING>(q, 2 * c + 1, w.cs, lg, a1, b1);
                const float va[8] = {a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]};
                const float vb[8] = {b0[0], b0[1], b0[2], b0[3], b1[0], b1[1], b1[2], b1[3]};
                uint4 ha, la, hb, lb;
                split8<DT>(va, ha, la);
                split8<DT>(vb, hb, lb);
#pragma unroll
                for (int tb = 0; tb < 2; ++tb) {
                    sc[rb][tb] = Mma<DT>::run(kf[tb][c], la, sc[rb][tb]);
                    sc[rb][tb] = Mma<DT>::run(kf[tb][2 + c], lb, sc[rb][tb]);
                    sc[rb][tb] = Mma<DT>::run(kf[tb][c], ha, sc[rb][tb]);
                    sc[rb][tb] = Mma<DT>::run(kf[tb][2 + c], hb, sc[rb][tb]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            const int last = min(cd.ntok - 1, st.trow[rb] - cd.tok0) - 4 * lg;
#pragma unroll
            for (int e = 0; e < 8; ++e) sc[rb][e >> 2][e & 3] = 16 * (e >> 2) + (e & 3) <= last ? sc[rb][e >> 2][e & 3] : -INFINITY;
        }
        float pv[NRB][8];
        st.softmax(sc, [&](int) { return a.scale_log2e; }, pv);
        st.template weigh<DT, true>(w.v_lds + (4 * lg + (li >> 2)) * kVRow + 8 * (li & 3), pv);
        wave_lds_order();                            // the next tile writes over what others read above
        // values that are not finite, for the rows that see them (zero times one would reach the rows ahead)
        for (; odd; odd &= odd - 1) {
            const int j = __builtin_ctz(odd);
#pragma unroll
            for (int db = 0; db < 8; ++db) {
                const auto x = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(rv, j * pitch + 32 * db + 8 * lg, 0, 0));
                const float v[4] = {Mma<DT>::lo(x.x), Mma<DT>::hi(x.x), Mma<DT>::lo(x.y), Mma<DT>::hi(x.y)};
#pragma unroll
                for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (cd.tok0 + j <= st.trow[rb] && !(fabsf(v[r]) < INFINITY)) st.acc[rb][db][r] += v[r];
            }
        }
        st.pin();
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
template <int DT, int PAIRING, bool REG_TABLE>
__global__ __launch_bounds__(kSoloThreads, 2) void attn_q4_solo_kernel(AttnArgs a, RopeFreq freq, Plan p, Scales s) {
    __shared__ std::conditional_t<REG_TABLE, int, SegTable> lds_tbl;
    __shared__ __attribute__((aligned(16))) unsigned char lds[kSoloWaves * kVTile];
    __shared__ __attribute__((aligned(16))) float2 cs_lds[kSoloWaves][64];
    __shared__ float2 red_ml[kSoloWaves][16];
    static_assert(kSoloWaves * kVTile >= kSoloWaves * 8 * kWave * (int)sizeof(f32x4), "the results reuse the V tiles");

    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int li = lane & 15, lg = lane >> 4;
    // grid (split, kv head, query)
    const int split = blockIdx.x, hkv = blockIdx.y, b = blockIdx.z;
    const int unit = b * p.units_per_b + hkv;
    const QueryHead qh = load_query_head(a, b, REG_TABLE ? lane : (int)threadIdx.x);
    const int tq = max(min(qh.tq_raw, a.max_tq), 0);
    Rows<1> st;
    st.begin(0, p.group * tq, p.group, a.n_q_heads, hkv, li);
    RegSegTable rtbl;
    int total;
    if constexpr (REG_TABLE) {
        rtbl = build_reg_table(a, qh, lane, kTile);
        total = rtbl.total;
    } else {
        build_table(a, qh, &lds_tbl, kTile);
        total = lds_tbl.tile0[lds_tbl.n];
    }
    char* const ws = static_cast<char*>(a.workspace);
    WavePlace w;
    w.li = li; w.lg = lg; w.hkv = hkv; w.rows_wg = p.rows_wg; w.ss = split * kSoloWaves + wave;
    w.t_begin = run_begin(total, p.nsplit * kSoloWaves, w.ss);
    w.t_end = run_begin(total, p.nsplit * kSoloWaves, w.ss + 1);
    w.q_first = (int64_t)qh.q0 * a.n_q_heads * kD;
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
    const QueryPart q = query_part(a, w, st, 0);
    const int q_scale = row_scale<DT>(q);
    const float down = scale_down(q_scale), mul = a.scale_log2e * scale_of((uint32_t)q_scale);
    unsigned char* const v_write = w.v_lds + li * kVRow + 64 * lg;
    const unsigned char* const v_read = w.v_lds + (4 * lg + (li >> 2)) * kVRow + 8 * (li & 3);
    Parts qt;
    int q_delta = 0;
    bool have_parts = false, passed_over = false;
    auto step = [&](Tile& d, TileRegs& r) __attribute__((always_inline)) {
        const Tile cd = d;
        // a tile that is passed over counts as one without tokens (no branch around the body: the compiler would keep the accumulators twice)
        const bool take = tile_fits(r, cd.ntok, li);
        const int ntok = take ? cd.ntok : 0;
        passed_over = passed_over || !take;
        st.enter(cd.seg, w.massml, w.rows_wg, w.ss, false, li, lg);
        if (!have_parts || cd.delta != q_delta) {
            have_parts = true;
            q_delta = cd.delta;
            put_angles(w.cs, lane, cd.delta, w.my_freq, 1.f);
            qt = to_parts<DT, PAIRING>(q, down, w.cs, lg);
        }
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                *reinterpret_cast<uint4*>(v_write + 16 * tb * kVRow + 16 * c) = unpack8<CF_F16>(r.v[tb][c], take ? scale_of(r.vs[tb]) : 0.f);
        wave_lds_order();
        f32x4 sc[1][2] = {{f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}}};
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) sc[0][tb] = mma_fp4(r.k[tb], (int)r.ks[tb], qt.lo, kLoScale, sc[0][tb]);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) sc[0][tb] = Mma<CF_F16>::run(unpack8<CF_F16>(r.k[tb][c], take ? scale_of(r.ks[tb]) : 0.f), qt.hi[c], sc[0][tb]);
        __builtin_amdgcn_sched_barrier(0);
        fetch(d, r);                                 // the registers are free again
        __builtin_amdgcn_sched_barrier(0);
        if (ntok < kTile) {
            const int lim = ntok - 4 * lg;
#pragma unroll
            for (int e = 0; e < 8; ++e) sc[0][e >> 2][e & 3] = 16 * (e >> 2) + (e & 3) < lim ? sc[0][e >> 2][e & 3] : -INFINITY;
        }
        float pv[1][8];
        st.softmax(sc, [&](int) { return mul; }, pv);
        st.template weigh<CF_F16, false>(v_read, pv);
        wave_lds_order();                            // the next step writes over what others read above
    };
    // (left from the middle: with a step skipped the wait for one register set would have to cover the other as well)
    while (d0.ntok > 0) {
        step(d0, r0);
        if (d1.ntok <= 0) break;
        step(d1, r1);
    }
    const bool own = walk.others;
    if (passed_over) with_table([&](const auto& t) __attribute__((always_inline)) { odd_tiles<DT, PAIRING, 1>(a, s, t, w, st); });
    if (own) with_table([&](const auto& t) __attribute__((always_inline)) { own_tiles<DT, PAIRING, 1>(a, t, w, st); });
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
// More row blocks: four wavefronts with NRB blocks each share 32-token tiles.  Bound by the instructions that a SIMD can issue.  Every thread
// loads 8 bytes of a tile's key codes and of its value codes, three tiles ahead of their use; the key codes go to LDS as they are (a
// wavefront unpacks them to its matrix operands), the values unpacked, each once per workgroup.  One barrier per tile.
template <int DT, int PAIRING, int NRB>
__global__ __launch_bounds__(kRowsThreads, NRB == 1 ? 3 : 2) void attn_q4_rows_kernel(AttnArgs a, RopeFreq freq, Plan p, Scales s) {
    constexpr int kKBuf = kTile * kRowBytes;
    __shared__ SegTable tbl;
    // two tiles' key codes, two of values, the workgroup's queries; after the last tile a V tile per wavefront
    constexpr int kTiles = 2 * (kKBuf + kVTile), kQueries = kRowsWaves * NRB * 16 * kQRow;
    constexpr int kRowsBytes = kTiles + kQueries > kRowsWaves * kVTile ? kTiles + kQueries : kRowsWaves * kVTile;
    __shared__ __attribute__((aligned(16))) unsigned char lds[kRowsBytes];
    __shared__ __attribute__((aligned(16))) float2 cs_lds[kRowsWaves][64];
    __shared__ uint32_t ks_lds[2][kTile];            // the keys' scale bytes, four of a token
    __shared__ int odd_lds[2];                       // number of the last tile in a buffer whose scales do not fit fp16
    __shared__ uint32_t top_lds;

    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int li = lane & 15, lg = lane >> 4;
    // grid (split, kv head * row groups + row group, query)
    const int split = blockIdx.x, b = blockIdx.z;
    const int hkv = p.n_rg == 1 ? (int)blockIdx.y : (int)div_exact(blockIdx.y, (unsigned)p.n_rg), rg = (int)blockIdx.y - hkv * p.n_rg;
    const int unit = b * p.units_per_b + (int)blockIdx.y;
    const QueryHead qh = load_query_head(a, b, tid);
    const int tq = max(min(qh.tq_raw, a.max_tq), 0);
    const int row0 = rg * p.rows_wg;
    const bool wg_rows = row0 < p.group * tq;        // workgroup-uniform
    Rows<NRB> st;
    st.begin(row0 + wave * NRB * 16, p.group * tq, p.group, a.n_q_heads, hkv, li);
    char* const ws = static_cast<char*>(a.workspace);
    WavePlace w;
    w.li = li; w.lg = lg; w.hkv = hkv; w.rows_wg = p.rows_wg; w.ss = split;
    w.q_first = (int64_t)qh.q0 * a.n_q_heads * kD;
    w.my_freq = freq.rev[lane];
    w.cs = cs_lds[wave];
    w.v_lds = lds + wave * kVTile;
    w.massml = a.mass ? reinterpret_cast<float2*>(ws + p.off_massml) + (int64_t)unit * p.slots * p.rows_wg + wave * NRB * 16 : nullptr;
    // the power of two that the workgroup's queries are scaled down by
    if (tid == 0) { top_lds = 0; odd_lds[0] = odd_lds[1] = -1; }
    uint32_t top = 0;
    unsigned char* const q_lds = lds + kTiles + (wave * NRB * 16 + li) * kQRow + 32 * lg;     // (a wavefront reads its own rows only)
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
        const QueryPart q = query_part(a, w, st, rb);
        top = max(top, largest<DT>(q));
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(q_lds + rb * 16 * kQRow + 128 * (i >> 1) + 16 * (i & 1)) = q.w[i];
    }
    build_table(a, qh, &tbl, kTile);                 // (its barriers are after the line above)
    atomicMax(&top_lds, top);
    const int total = wg_rows ? tbl.tile0[tbl.n] : 0;
    w.t_begin = run_begin(total, p.nsplit, split);
    w.t_end = run_begin(total, p.nsplit, split + 1);

    RunWalk<false> walk(w.t_begin, w.t_end);
    const int row_bytes = (int)(a.store_ts >> 1), scale_bytes = (int)(a.store_ts >> 5);
    const int st_tok = tid >> 3, st_part = tid & 7;  // token and 16 channels that the thread stages
    struct Regs { uint2 k, v; uint32_t vs, ks; };
    auto fetch = [&](Tile& d, Regs& r) __attribute__((always_inline)) {
        d = walk.next(tbl, lane);
        const bool any = d.ntok > 0;
        const int64_t at = any ? (walk.c_tok + d.tok0) * a.store_ts + (int64_t)hkv * a.store_hs : 0;
        const int codes = any ? (d.ntok - 1) * row_bytes + kRowBytes : 0, scales = any ? (d.ntok - 1) * scale_bytes + 4 : 0;
        const int off = st_tok * row_bytes + 8 * st_part;
        r.k = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(buffer(a.k_store, at >> 1, codes), off, 0, 0));
        r.v = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(buffer(a.v_store, at >> 1, codes), off, 0, 0));
        r.vs = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(buffer(s.v, at >> 5, scales), st_tok * scale_bytes + (st_part >> 1), 0, 0);
        r.ks = __builtin_amdgcn_raw_buffer_load_b32(buffer(s.k, at >> 5, scales), (lane & 31) * scale_bytes, 0, 0);
    };
    auto stage = [&](const Tile& d, const Regs& r, int buf, int number) __attribute__((always_inline)) {
        unsigned char* const k_buf = lds + buf * kKBuf;
        unsigned char* const v_buf = lds + 2 * kKBuf + buf * kVTile;
        *reinterpret_cast<uint2*>(k_buf + 8 * tid) = r.k;
        const bool fits = fits_f16(r.vs);
        const float sv = fits ? scale_of(r.vs) : 0.f;
        unsigned char* const to = v_buf + st_tok * kVRow + 32 * st_part;
        *reinterpret_cast<uint4*>(to) = unpack8<CF_F16>(r.v.x, sv);
        *reinterpret_cast<uint4*>(to + 16) = unpack8<CF_F16>(r.v.y, sv);
        if (tid < kTile) ks_lds[buf][tid] = r.ks;
        const bool k_fits = fits_f16(r.ks & 255) && fits_f16(r.ks >> 8 & 255) && fits_f16(r.ks >> 16 & 255) && fits_f16(r.ks >> 24);
        if ((!fits && st_tok < d.ntok) || (!k_fits && tid < d.ntok)) odd_lds[buf] = number;
    };

    Tile dc, dn;
    Regs r;
    fetch(dc, r);
    __syncthreads();                                 // top_lds
    const int q_scale = scale_byte_of<DT>(top_lds);
    const float down = scale_down(q_scale), mul = a.scale_log2e * scale_of((uint32_t)q_scale);
    // two tables of angles, of the current and of the next segment's tiles, times `down`
    int cs_slot = 0;
    auto angles = [&](int slot, int delta) __attribute__((always_inline)) {
        if (wave == 0) {
            const float2 c = rope_cos_sin_fast(delta, w.my_freq);
            cs_lds[slot][lane] = make_float2(c.x * down, c.y * down);
        }
    };
    angles(0, dc.delta);
    stage(dc, r, 0, 0);
    fetch(dn, r);
    Parts qt[NRB];
    int q_delta = 0, number = 0;
    bool have_parts = false, passed_over = false;
    const unsigned char* const v_read = lds + 2 * kKBuf + (4 * lg + (li >> 2)) * kVRow + 8 * (li & 3);
    // Step: tile `dc` is in buffer `buf`; the one after it, dn, is on its way to registers since a step ago, from where it goes to the other
    // buffer, and the next one is requested.  (Two sets of registers, two tiles ahead: the compiler waits for both at the loop's head.)
    for (int buf = 0; dc.ntok > 0; buf ^= 1, ++number) {
        __syncthreads();                             // tile `dc` is staged; every wavefront is done with the other buffer
        const Tile cd = dc;
        const bool turn_next = dn.ntok > 0 && dn.delta != cd.delta;
        const int next_delta = dn.delta;
        dc = dn;
        stage(dn, r, buf ^ 1, number + 1);
        fetch(dn, r);
        const bool take = odd_lds[buf] != number;
        i32x4 kc[2];
        uint32_t ks[2];
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            kc[tb] = *reinterpret_cast<const i32x4*>(lds + buf * kKBuf + (16 * tb + li) * kRowBytes + 16 * lg);
            ks[tb] = reinterpret_cast<const uint8_t*>(ks_lds[buf])[4 * (16 * tb + li) + lg];
        }
        st.enter(cd.seg, w.massml, w.rows_wg, w.ss, false, li, lg);
        if (!have_parts || cd.delta != q_delta) {
            have_parts = true;
            q_delta = cd.delta;
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) {
                QueryPart q;
#pragma unroll
                for (int i = 0; i < 4; ++i) q.w[i] = *reinterpret_cast<const uint4*>(q_lds + rb * 16 * kQRow + 128 * (i >> 1) + 16 * (i & 1));
                qt[rb] = to_parts<DT, PAIRING>(q, 1.f, cs_lds[cs_slot], lg);
            }
        }
        if (turn_next) {
            cs_slot ^= 1;
            angles(cs_slot, next_delta);
        }
        const int ntok = take ? cd.ntok : 0;
        passed_over = passed_over || !take;
        f32x4 sc[NRB][2];
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) sc[rb][tb] = mma_fp4(kc[tb], (int)ks[tb], qt[rb].lo, kLoScale, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) {
                const uint4 kf = unpack8<CF_F16>(kc[tb][c], scale_of(ks[tb]));
#pragma unroll
                for (int rb = 0; rb < NRB; ++rb) sc[rb][tb] = Mma<CF_F16>::run(kf, qt[rb].hi[c], sc[rb][tb]);
            }
        if (ntok < kTile) {
            const int lim = ntok - 4 * lg;
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                for (int e = 0; e < 8; ++e) sc[rb][e >> 2][e & 3] = 16 * (e >> 2) + (e & 3) < lim ? sc[rb][e >> 2][e & 3] : -INFINITY;
        }
        float pv[NRB][8];
        st.softmax(sc, [&](int) { return mul; }, pv);
        st.template weigh<CF_F16, false>(v_read + buf * kVTile, pv);
    }
    const bool own = walk.others;
    __syncthreads();                                 // the buffers become the wavefronts' own
    if (passed_over) odd_tiles<DT, PAIRING, NRB>(a, s, tbl, w, st);
    if (own) own_tiles<DT, PAIRING, NRB>(a, tbl, w, st);
    st.emit(w.massml, w.rows_wg, w.ss, false, li, lg);
    st.close();
    const int64_t part = (int64_t)unit * p.nsplit + split;
    float2* const ml = reinterpret_cast<float2*>(ws + p.off_ml) + part * p.rows_wg + wave * NRB * 16;
    float* const opart = reinterpret_cast<float*>(ws + p.off_opart) + (part * p.rows_wg + wave * NRB * 16) * kD;
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
}

// ---------------------------------------------------------------------------------------------
// Merges the splits' partial rows, a wavefront per row: lane s holds the statistics of split s, then a lane two channels.  A row's own
// (maximum, sum) replaces split 0's, for the mass kernel.
template <int DT>
__global__ __launch_bounds__(256) void q4_combine_kernel(AttnArgs a, Plan p) {
    const int b = blockIdx.z, unit = b * p.units_per_b + (int)blockIdx.y;
    const int hkv = p.n_rg == 1 ? (int)blockIdx.y : (int)div_exact(blockIdx.y, (unsigned)p.n_rg), rg = (int)blockIdx.y - hkv * p.n_rg;
    const int lane = threadIdx.x & (kWave - 1);
    const int row = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + (int)threadIdx.x / kWave);
    char* ws = static_cast<char*>(a.workspace);
    const int64_t first = (int64_t)unit * p.nsplit * p.rows_wg + row;
    float2* const ml = reinterpret_cast<float2*>(ws + p.off_ml) + first;
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
    const float l = wave_sum(weight);
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
    if (a.mass && lane == 0) ml[0] = make_float2(mx, l);
}

// Per-segment attention mass, a workgroup per table entry: over the units, the runs that hold the segment's tiles and the rows, sum * exp2(reference -
// row maximum) / row sum, in a fixed order.  Then S += mass (Alg. 2): a document slot's first entry works out the masses of all of the slot's
// entries and adds them up in table order.
__global__ __launch_bounds__(256) void q4_mass_kernel(AttnArgs a, Plan p) {
    __shared__ SegTable tbl;
    __shared__ float part_sum[4];
    const int b = blockIdx.y, entry = blockIdx.x, tid = threadIdx.x;
    const QueryHead qh = load_query_head(a, b, tid);
    build_table(a, qh, &tbl, kTile);
    if (entry >= tbl.n) return;
    const char* ws = static_cast<const char*>(a.workspace);
    const int tq = max(min(qh.tq_raw, a.max_tq), 0), n_rows = p.group * tq;
    const int total = tbl.tile0[tbl.n], nsub = p.nsplit * p.runs;
    auto mass_of = [&](int s) {
        const int ts = tbl.tile0[s], te = tbl.tile0[s + 1];
        float sum = 0.f;
        if (te > ts) {
            const int sub0 = run_of(total, nsub, ts), sub1 = run_of(total, nsub, te - 1);
            const int n_sub = sub1 - sub0 + 1;
            // items: unit, run, row; threads take rows of one (unit, run) side by side
            const int rows = min(p.rows_wg, 256), per = 256 / rows;      // rows_wg is a power of two
            const int row = tid & (rows - 1), first = tid / rows;
            for (int i = first; i < p.units_per_b * n_sub; i += per) {
                const int u = (int)div_exact((unsigned)i, (unsigned)n_sub), sub = sub0 + i - u * n_sub;
                // a run between a segment's first and last may own no tile at all: its slot was not written
                if (run_begin(total, nsub, sub) >= run_begin(total, nsub, sub + 1)) continue;
                const int rg = u - (int)div_exact((unsigned)u, (unsigned)p.n_rg) * p.n_rg;
                const int64_t unit = (int64_t)b * p.units_per_b + u;
                if (rg * p.rows_wg + row >= n_rows) continue;
                const float2 v = reinterpret_cast<const float2*>(ws + p.off_massml)[(unit * p.slots + s + sub) * p.rows_wg + row];
                const float2 r = reinterpret_cast<const float2*>(ws + p.off_ml)[unit * p.nsplit * p.rows_wg + row];
                const float m = r.x == -INFINITY ? 0.f : r.x;
                sum += v.y * __builtin_amdgcn_exp2f(v.x - m) * (r.y > 0.f ? 1.f / r.y : r.y);
            }
        }
        sum = wave_sum(sum);
        __syncthreads();
        if ((tid & (kWave - 1)) == 0) part_sum[tid / kWave] = sum;
        __syncthreads();
        return ((part_sum[0] + part_sum[1]) + part_sum[2]) + part_sum[3];
    };
    const float mine = mass_of(entry);
    if (tid == 0) a.mass[(int64_t)b * a.seg_stride + entry] = mine;
    if (a.score_accum == nullptr) return;
    const int d = tbl.doc[entry];
    if (d < 0 || d >= a.score_stride) return;
    float sum = mine;
    for (int j = 0; j < tbl.n; ++j) {                // workgroup-uniform
        if (tbl.doc[j] != d) continue;
        if (j < entry) return;
        if (j > entry) sum += mass_of(j);
    }
    if (tid == 0) a.score_accum[(int64_t)b * a.score_stride + d] += sum;
}

}  // namespace
}  // namespace q4

size_t q4_workspace_bytes(const cf_layer_desc* d, int32_t batch, int32_t max_tq, int32_t seg_stride, int64_t max_kv_tokens) {
    return q4::make_plan(d->n_q_heads, d->n_kv_heads, batch, max_tq, seg_stride, max_kv_tokens).total;
}

cf_status launch_attention_q4(const AttnArgs& a, const q4::Scales& sc, const RopeFreq& f, hipStream_t s) {
    using namespace q4;
    const Plan p = make_plan(a.n_q_heads, a.n_kv_heads, a.batch, a.max_tq, a.seg_stride, a.max_kv_tokens);
    if (a.batch > 65535 || p.units_per_b > 65535) {
        set_error("neither batch nor n_kv_heads * row groups may exceed 65535 on this path");
        return CF_ERR_UNSUPPORTED;
    }
    const dim3 grid((unsigned)p.nsplit, (unsigned)p.units_per_b, (unsigned)a.batch);
    auto go = [&](auto dt, auto pairing) {
        constexpr int DT = decltype(dt)::value, PAIRING = decltype(pairing)::value;
        if (p.solo) {
            if (a.seg_stride <= kWave) hipLaunchKernelGGL((attn_q4_solo_kernel<DT, PAIRING, true>), grid, dim3(kSoloThreads), 0, s, a, f, p, sc);
            else hipLaunchKernelGGL((attn_q4_solo_kernel<DT, PAIRING, false>), grid, dim3(kSoloThreads), 0, s, a, f, p, sc);
        } else if (p.nrb == 1) {
            hipLaunchKernelGGL((attn_q4_rows_kernel<DT, PAIRING, 1>), grid, dim3(kRowsThreads), 0, s, a, f, p, sc);
        } else {
            hipLaunchKernelGGL((attn_q4_rows_kernel<DT, PAIRING, 2>), grid, dim3(kRowsThreads), 0, s, a, f, p, sc);
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
    if (!p.direct_out) {
        const dim3 rows((unsigned)p.rows_wg / 4, (unsigned)p.units_per_b, (unsigned)a.batch);
        if (bf16) hipLaunchKernelGGL(q4_combine_kernel<CF_BF16>, rows, dim3(256), 0, s, a, p);
        else hipLaunchKernelGGL(q4_combine_kernel<CF_F16>, rows, dim3(256), 0, s, a, p);
        CF_HIP(hipGetLastError());
    }
    if (a.mass != nullptr) {
        hipLaunchKernelGGL(q4_mass_kernel, dim3((unsigned)a.seg_stride, (unsigned)a.batch), dim3(256), 0, s, a, p);
        CF_HIP(hipGetLastError());
    }
    return CF_OK;
}

}  // namespace cf
