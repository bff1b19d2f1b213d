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
// Work: the rows that share a kv head (row m = t * group + head) are cut into 16-row blocks, one or two per wavefront.  A workgroup's eight wavefronts
// own different rows, or stream different runs of the 32-token tiles where there are few rows, or both; none waits for another
// before the end, where runs meet in LDS.  Splits (workgroups of the same rows) leave fp32 partial rows that a second kernel merges.
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

constexpr int kThreads = kWaves * kWave;
constexpr int kVRow = 288;                           // bytes per token of a staged V tile
constexpr int kVTile = kTile * kVRow;
constexpr int kRowBytes = 64;                        // codes of a row
constexpr float kProbLimit = attn::kProbLimit;

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// run i of a list of `total` tiles owns [total*i/n, total*(i+1)/n)
__device__ __forceinline__ int run_begin(int total, int n, int i) { return (int)((int64_t)total * i / n); }

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
__device__ __forceinline__ void turn4(const QueryPart& q, int n, bool still, const float2* cs, int lg, float (&a)[4], float (&b)[4]) {
    const uint4 wa = q.w[n >> 1], wb = q.w[2 + (n >> 1)];
    const uint32_t ua[2] = {n & 1 ? wa.z : wa.x, n & 1 ? wa.w : wa.y}, ub[2] = {n & 1 ? wb.z : wb.x, n & 1 ? wb.w : wb.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = i & 1 ? Mma<DT>::hi(ua[i >> 1]) : Mma<DT>::lo(ua[i >> 1]);
        b[i] = i & 1 ? Mma<DT>::hi(ub[i >> 1]) : Mma<DT>::lo(ub[i >> 1]);
    }
    if (still) return;                               // wavefront-uniform
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

// The exponent byte of a row's power of two: its largest channel, turned by any angle, comes to at most 2^7 * sqrt(2) of it; 255 (NaN) for a
// row that is not finite.
template <int DT>
__device__ __forceinline__ int row_scale(const QueryPart& q) {
    uint32_t top = 0;                                // magnitudes as bits: a NaN counts as the largest
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t u[4] = {q.w[i].x, q.w[i].y, q.w[i].z, q.w[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) top = max(top, max(u[j] & 0x7fffu, u[j] >> 16 & 0x7fffu));
    }
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    if (top >= (DT == CF_BF16 ? 0x7f80u : 0x7c00u)) return 255;
    const float t = Mma<DT>::lo(top);
    return max((int)(__float_as_uint(t) >> 23) - 6, 27);
}

__device__ __forceinline__ float scale_down(int scale) { return __uint_as_float((uint32_t)(254 - min(scale, 253)) << 23); }

// A 16-row block of turned queries: fp16 values (hi[s]: channels 32 lg + 8 s .. + 7) and what is left, 2^11 times larger, in e4m3.
constexpr int kLoScale = 127 - 11;
struct Parts { uint4 hi[4]; i32x8 lo; };

// `lds`: the wavefront's staging rows.  A lane turns channels 16 lg .. and 64 + 16 lg .. (both of a slice), the fp16 fragments want 32 lg ...
template <int DT, int PAIRING>
__device__ __forceinline__ Parts to_parts(const QueryPart& q, int scale, bool still, const float2* cs, unsigned char* lds, int li, int lg) {
    const float down = scale_down(scale);
    Parts r;
    auto split = [&](float (&v)[4], int w, unsigned char* at) __attribute__((always_inline)) {
        const uint32_t h0 = Mma<CF_F16>::pack(v[0] * down, v[1] * down), h1 = Mma<CF_F16>::pack(v[2] * down, v[3] * down);
        *reinterpret_cast<uint2*>(at) = make_uint2(h0, h1);
        auto rest = [&](int i, float h) { return fmaf(v[i], down, -h) * 2048.f; };       // exact
        const int packed = __builtin_amdgcn_cvt_pk_fp8_f32(rest(0, Mma<CF_F16>::lo(h0)), rest(1, Mma<CF_F16>::hi(h0)), 0, false);
        r.lo[w] = __builtin_amdgcn_cvt_pk_fp8_f32(rest(2, Mma<CF_F16>::lo(h1)), rest(3, Mma<CF_F16>::hi(h1)), packed, true);
    };
    unsigned char* const write = lds + li * kVRow + 32 * lg;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        float a[4], b[4];
        turn4<DT, PAIRING>(q, n, still, cs, lg, a, b);
        split(a, n, write + 8 * n);
        split(b, 4 + n, write + 128 + 8 * n);
        __builtin_amdgcn_sched_barrier(0);           // few floats at a time
    }
    wave_lds_order();
#pragma unroll
    for (int s = 0; s < 4; ++s) r.hi[s] = *reinterpret_cast<const uint4*>(lds + li * kVRow + 64 * lg + 16 * s);
    wave_lds_order();
    return r;
}

// The same as three terms of e4m3, 16 times larger from one to the next, for keys of any scale.
constexpr int kTerms = 3;
struct Terms { i32x8 t[kTerms]; };

template <int DT, int PAIRING>
__device__ __forceinline__ Terms to_terms(const QueryPart& q, int scale, bool still, const float2* cs, int lg) {
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
        turn4<DT, PAIRING>(q, n, still, cs, lg, a, b);
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

template <int DT, int PAIRING, int NRB, bool REG_TABLE>
__global__ __launch_bounds__(kThreads, 2) void attn_q4_kernel(AttnArgs a, RopeFreq freq, Plan p, Scales s) {
    __shared__ std::conditional_t<REG_TABLE, int, SegTable> tbl;
    constexpr int kMerge = kWaves * 8 * kWave * (int)sizeof(f32x4);
    __shared__ __attribute__((aligned(16))) unsigned char lds[kWaves * kVTile > kMerge ? kWaves * kVTile : kMerge];
    __shared__ __attribute__((aligned(16))) float2 cs_lds[kWaves][64];
    __shared__ float2 red_ml[kWaves][NRB * 16];

    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int li = lane & 15, lg = lane >> 4;
    // grid (split, kv head * row groups + row group, query)
    const int split = blockIdx.x, b = blockIdx.z;
    const int hkv = (int)div_exact(blockIdx.y, (unsigned)p.n_rg), rg = (int)blockIdx.y - hkv * p.n_rg;
    const int unit = b * p.units_per_b + (int)blockIdx.y;
    const int row_wave = wave & (p.row_waves - 1), run = (int)div_exact((unsigned)wave, (unsigned)p.row_waves);
    const int group = p.group;
    const QueryHead qh = load_query_head(a, b, REG_TABLE ? lane : (int)threadIdx.x);
    const double my_freq = freq.rev[lane];
    const int tq = max(min(qh.tq_raw, a.max_tq), 0);
    const int n_rows = group * tq;
    const int row0 = rg * p.rows_wg + row_wave * NRB * 16;       // the wavefront's first row

    RegSegTable rtbl;
    int total;
    if constexpr (REG_TABLE) {
        rtbl = build_reg_table(a, qh, lane, kTile);
        total = rtbl.total;
    } else {
        build_table(a, qh, &tbl, kTile);
        total = tbl.tile0[tbl.n];
    }
    const int nsub = p.nsplit * p.runs, ss = split * p.runs + run;
    const bool has_rows = row0 < n_rows;             // wavefront-uniform
    const int t_begin = run_begin(total, nsub, ss), t_end = has_rows ? run_begin(total, nsub, ss + 1) : 0;
    RunWalk<false> walk(t_begin, t_end);

    // row m = t * group + head
    int trow[NRB], qrow[NRB];                        // place in the own block (-1: no row); row of q and out, counted from the query's first
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
        const int m = row0 + 16 * rb + li;
        const bool valid = m < n_rows;
        const int t = valid ? (int)div_exact((unsigned)m, (unsigned)group) : 0, g = valid ? m - t * group : 0;
        trow[rb] = valid ? t : -1;
        qrow[rb] = t * a.n_q_heads + hkv * group + g;
    }
    const int64_t q_first = (int64_t)qh.q0 * a.n_q_heads * kD;
    auto query = [&](int rb) {
        int row = qrow[rb];
        asm volatile("" : "+v"(row));                // its addresses are worked out anew, not kept through the loops
        return load_query(static_cast<const uint16_t*>(a.q) + q_first + (int64_t)row * kD, trow[rb] >= 0, lg);
    };

    int q_scale[NRB];
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) q_scale[rb] = row_scale<DT>(query(rb));

    // One tile's codes and scales: token 16 tb + li, 32 channels from 32 lg on.
    struct Regs { i32x4 k[2], v[2]; uint32_t ks[2], vs[2]; };
    const int row_bytes = (int)(a.store_ts >> 1), scale_bytes = (int)(a.store_ts >> 5);
    auto fetch = [&](RunWalk<false>& walk, Tile& d, Regs& r) {
        if constexpr (REG_TABLE) d = walk.next(rtbl, lane);
        else d = walk.next(tbl, lane);
        // rows past a ragged tile's end, and everything where no tile of the store is left, lie past the range and read as zero
        const bool any = d.ntok > 0;
        const int64_t at = any ? (walk.c_tok + d.tok0) * a.store_ts + (int64_t)hkv * a.store_hs : 0;
        const int codes = any ? (d.ntok - 1) * row_bytes + kRowBytes : 0, scales = any ? (d.ntok - 1) * scale_bytes + 4 : 0;
        auto rsrc = [](const void* base, int64_t off, int range) {
            return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(base) + off), 0, range, 0x00020000);
        };
        const auto rk = rsrc(a.k_store, at >> 1, codes), rv = rsrc(a.v_store, at >> 1, codes);
        const auto sk = rsrc(s.k, at >> 5, scales), sv = rsrc(s.v, at >> 5, scales);
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
            const int off = (16 * tb + li) * row_bytes + 16 * lg, soff = (16 * tb + li) * scale_bytes + lg;
            r.k[tb] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, off, 0, 0));
            r.v[tb] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, off, 0, 0));
            r.ks[tb] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(sk, soff, 0, 0);
            r.vs[tb] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(sv, soff, 0, 0);
        }
    };

    f32x4 acc[NRB][8];
    float m_run[NRB], l_run[NRB], seg_l[NRB];
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
#pragma unroll
        for (int db = 0; db < 8; ++db) acc[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
        m_run[rb] = -INFINITY;
        l_run[rb] = seg_l[rb] = 0.f;
    }
    char* const ws = static_cast<char*>(a.workspace);
    float2* const massml = reinterpret_cast<float2*>(ws + p.off_massml) + (int64_t)unit * p.slots * p.rows_wg + row_wave * NRB * 16;
    const bool want_mass = a.mass != nullptr;
    // what scores are multiplied by: of whole queries, and of those scaled down by their row's power of two
    const float scale_log2e = a.scale_log2e;
    auto plain_mul = [&](int) { return scale_log2e; };
    auto part_mul = [&](int rb) { return scale_log2e * scale_of((uint32_t)q_scale[rb]); };
    unsigned char* const v_lds = lds + wave * kVTile;
    unsigned char* const v_write = v_lds + li * kVRow + 64 * lg;
    const unsigned char* const v_read = v_lds + (4 * lg + (li >> 2)) * kVRow + 8 * (li & 3);

    // (reference, sum) per row of the segment that ends here; `again`: added to what its slot holds, whose reference is not larger
    bool again = false;
    auto emit = [&](int seg) {
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            float tot = seg_l[rb] + __shfl_xor(seg_l[rb], 16);
            tot += __shfl_xor(tot, 32);
            if (lg == 0) {
                float2* slot = massml + (int64_t)(seg + ss) * p.rows_wg + 16 * rb + li;
                if (again && slot->x != -INFINITY) tot += slot->y * __builtin_amdgcn_exp2f(slot->x - m_run[rb]);
                *slot = make_float2(m_run[rb], tot);
            }
        }
    };
    // Online softmax (exp2 domain) of scores sc, in units of `mul` per row, against a stale row maximum: probabilities pv; see kProbLimit.
    auto softmax = [&](f32x4 (&sc)[NRB][2], auto mul, float (&pv)[NRB][8]) {
        float lsum[NRB];
        auto probabilities = [&](int rb) {
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
        // (one place for the accumulators: the compiler would keep a copy for either way through the branch)
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
            for (int db = 0; db < 8; ++db) asm volatile("" : "+v"(acc[rb][db]));
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
            l_run[rb] += lsum[rb];
            seg_l[rb] += lsum[rb];
        }
    };
    // O^T += V^T P^T; VT: the type V is staged in.  `exact`: P as value and remainder.
    auto weigh = [&](auto vt, auto exact, const float (&pv)[NRB][8]) {
        constexpr int VT = decltype(vt)::value;
        uint4 ph[NRB], pl[NRB];
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) split8<VT>(pv[rb], ph[rb], pl[rb]);
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            if (NRB > 1 && (db & 3) == 0) __builtin_amdgcn_sched_barrier(0);     // half of V^T in registers
            const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)(v_read + 32 * db));
            const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((short4v __attribute__((address_space(3)))*)(v_read + 32 * db + 16 * kVRow));
            const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
            const uint4 va = make_uint4(l2.x, l2.y, h2.x, h2.y);
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) {
                if constexpr (decltype(exact)::value) acc[rb][db] = Mma<VT>::run(va, pl[rb], acc[rb][db]);
                acc[rb][db] = Mma<VT>::run(va, ph[rb], acc[rb][db]);
            }
        }
    };

    int cs_delta = 0, cur_seg = -1;
    auto angles = [&](int delta) {                   // the wavefront's table of (cos, sin)
        if (delta == 0 || delta == cs_delta) return;
        cs_delta = delta;
        wave_lds_order();
        cs_lds[wave][lane] = rope_cos_sin_fast(delta, my_freq);
        wave_lds_order();
    };
    auto enter = [&](int seg) {
        if (seg == cur_seg) return;
        if (want_mass && cur_seg >= 0) emit(cur_seg);
        cur_seg = seg;
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) seg_l[rb] = 0.f;
    };

    // ---- the run's tiles of the store.  `wide` false: those whose values fit fp16, the others are passed over; true: the others, with values and
    // probabilities in bf16 (the latter as value and remainder).
    bool passed_over = false;
    auto store_tiles = [&](auto wide, RunWalk<false>& walk, Tile d, Regs& r) {
        constexpr int VT = decltype(wide)::value ? CF_BF16 : CF_F16;
        std::conditional_t<decltype(wide)::value, Terms, Parts> qt[NRB];
        int q_delta = 0;
        bool have_terms = false;
        while (d.ntok > 0) {
            const Tile cd = d;
            const bool fits = __all(((fits_f16(r.ks[0]) && fits_f16(r.vs[0])) || li >= cd.ntok) &&
                                    ((fits_f16(r.ks[1]) && fits_f16(r.vs[1])) || 16 + li >= cd.ntok));
            // a tile that is passed over counts as one without tokens (no branch around the body: the compiler would keep the accumulators twice)
            const bool take = fits != decltype(wide)::value;
            const int ntok = take ? cd.ntok : 0;
            passed_over = passed_over || !take;
            enter(cd.seg);
            if (!have_terms || cd.delta != q_delta) {
                have_terms = true;
                q_delta = cd.delta;
                angles(cd.delta);
#pragma unroll
                for (int rb = 0; rb < NRB; ++rb) {
                    const QueryPart q = query(rb);
                    if constexpr (decltype(wide)::value) qt[rb] = to_terms<DT, PAIRING>(q, q_scale[rb], cd.delta == 0, cs_lds[wave], lg);
                    else qt[rb] = to_parts<DT, PAIRING>(q, q_scale[rb], cd.delta == 0, cs_lds[wave], v_lds, li, lg);
                }
            }
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    *reinterpret_cast<uint4*>(v_write + 16 * tb * kVRow + 16 * c) = unpack8<VT>(r.v[tb][c], take ? scale_of(r.vs[tb]) : 0.f);
            wave_lds_order();
            f32x4 sc[NRB][2];
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) sc[rb][0] = sc[rb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (decltype(wide)::value) {
#pragma unroll
                for (int k = kTerms - 1; k >= 0; --k)        // the smallest terms first
#pragma unroll
                    for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                        for (int tb = 0; tb < 2; ++tb)
                            sc[rb][tb] = mma_fp4(r.k[tb], (int)r.ks[tb], qt[rb].t[k], q_scale[rb] == 255 ? 255 : q_scale[rb] - 4 * k, sc[rb][tb]);
            } else {
#pragma unroll
                for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                    for (int tb = 0; tb < 2; ++tb) sc[rb][tb] = mma_fp4(r.k[tb], (int)r.ks[tb], qt[rb].lo, kLoScale, sc[rb][tb]);
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int tb = 0; tb < 2; ++tb) {
                        const uint4 kf = unpack8<CF_F16>(r.k[tb][c], take ? scale_of(r.ks[tb]) : 0.f);
#pragma unroll
                        for (int rb = 0; rb < NRB; ++rb) sc[rb][tb] = Mma<CF_F16>::run(kf, qt[rb].hi[c], sc[rb][tb]);
                    }
            }
            fetch(walk, d, r);                       // the registers are free again
            if (ntok < kTile) {
                const int lim = ntok - 4 * lg;
#pragma unroll
                for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sc[rb][e >> 2][e & 3] = 16 * (e >> 2) + (e & 3) < lim ? sc[rb][e >> 2][e & 3] : -INFINITY;
            }
            float pv[NRB][8];
            if constexpr (decltype(wide)::value) softmax(sc, plain_mul, pv);
            else softmax(sc, part_mul, pv);
            weigh(std::integral_constant<int, VT>{}, wide, pv);
            wave_lds_order();                        // the next step writes over what others read above
        }
    };
    {
        Tile d;
        Regs r;
        fetch(walk, d, r);
        store_tiles(std::false_type{}, walk, d, r);
    }
    const bool own_tiles = walk.others;
    if (passed_over) {
        if (want_mass && cur_seg >= 0) emit(cur_seg);
        cur_seg = -1;
        again = true;                                // the segments' slots hold sums already
        RunWalk<false> rest(t_begin, t_end);
        Tile d;
        Regs r;
        fetch(rest, d, r);
        store_tiles(std::true_type{}, rest, d, r);
        if (want_mass && cur_seg >= 0) emit(cur_seg);
        cur_seg = -1;
        again = false;
    }
    // ---- its tiles of the own block: 16-bit keys and values, row t sees tokens 0 .. t
    if (own_tiles) {
        RunWalk<true> own(t_begin, t_end);
        for (;;) {
            Tile cd;
            if constexpr (REG_TABLE) cd = own.next(rtbl, lane);
            else cd = own.next(tbl, lane);
            if (cd.ntok <= 0) break;
            enter(cd.seg);
            angles(cd.delta);
            const int64_t at = ((own.c_tok + cd.tok0) * a.n_kv_heads + hkv) * kD * 2;
            const int pitch = a.n_kv_heads * kD * 2, range = (cd.ntok - 1) * pitch + 2 * kD;
            const auto rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(a.k_self) + at), 0, range, 0x00020000);
            const auto rv = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(a.v_self) + at), 0, range, 0x00020000);
            uint4 kf[2][4];
            uint32_t odd = 0;                        // tokens with values that are not finite
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) {
                bool any = false;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    kf[tb][c] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rk, (16 * tb + li) * pitch + 32 * lg + 128 * (c >> 1) + 16 * (c & 1), 0, 0));
                    const uint4 v = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rv, (16 * tb + li) * pitch + 64 * lg + 16 * c, 0, 0));
                    *reinterpret_cast<uint4*>(v_write + 16 * tb * kVRow + 16 * c) = finite8<DT>(v, any);
                }
                const uint64_t at = __ballot(any);
                odd |= (uint32_t)((at | at >> 16 | at >> 32 | at >> 48) & 0xffff) << (16 * tb);
            }
            wave_lds_order();
            f32x4 sc[NRB][2];
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) {
                const QueryPart q = query(rb);
                sc[rb][0] = sc[rb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < 2; ++c) {        // channels 8c .. 8c + 7 of either half
                    float a0[4], b0[4], a1[4], b1[4];
                    turn4<DT, PAIRING>(q, 2 * c, cd.delta == 0, cs_lds[wave], lg, a0, b0);
                    turn4<DT, PAIRING>(q, 2 * c + 1, cd.delta == 0, cs_lds[wave], lg, a1, b1);
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
                const int last = min(cd.ntok - 1, trow[rb] - cd.tok0) - 4 * lg;
#pragma unroll
                for (int e = 0; e < 8; ++e) sc[rb][e >> 2][e & 3] = 16 * (e >> 2) + (e & 3) <= last ? sc[rb][e >> 2][e & 3] : -INFINITY;
            }
            float pv[NRB][8];
            softmax(sc, plain_mul, pv);
            weigh(std::integral_constant<int, DT>{}, std::true_type{}, pv);
            wave_lds_order();                        // the next tile writes over what others read above
            // values that are not finite, for the rows that see them (zero times one would reach the rows ahead)
            for (; odd; odd &= odd - 1) {
                const int j = __builtin_ctz(odd);
#pragma unroll
                for (int db = 0; db < 8; ++db) {
                    const auto w = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(rv, j * pitch + 32 * db + 8 * lg, 0, 0));
                    const float v[4] = {Mma<DT>::lo(w.x), Mma<DT>::hi(w.x), Mma<DT>::lo(w.y), Mma<DT>::hi(w.y)};
#pragma unroll
                    for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (cd.tok0 + j <= trow[rb] && !(fabsf(v[r]) < INFINITY)) acc[rb][db][r] += v[r];
                }
            }
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                for (int db = 0; db < 8; ++db) asm volatile("" : "+v"(acc[rb][db]));
        }
    }
    if (want_mass && cur_seg >= 0) emit(cur_seg);

    // ---- the runs of the same rows meet: wavefront `run` takes the channel blocks run, run + runs, ...
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
        l_run[rb] += __shfl_xor(l_run[rb], 16);
        l_run[rb] += __shfl_xor(l_run[rb], 32);
        if (lg == 0) red_ml[wave][16 * rb + li] = make_float2(m_run[rb], l_run[rb]);
    }
    f32x4* const red = reinterpret_cast<f32x4*>(lds);
    const int64_t part = (int64_t)unit * p.nsplit + split;
    float2* const ml = reinterpret_cast<float2*>(ws + p.off_ml) + part * p.rows_wg + row_wave * NRB * 16;
    float* const opart = reinterpret_cast<float*>(ws + p.off_opart) + (part * p.rows_wg + row_wave * NRB * 16) * kD;
    auto meet = [&](auto block) {
        constexpr int rb = decltype(block)::value;
        __syncthreads();                             // nobody reads a V tile, or the block before, any more
#pragma unroll
        for (int db = 0; db < 8; ++db) red[(wave * 8 + db) * kWave + lane] = acc[rb][db];
        __syncthreads();
        float m = -INFINITY;
        for (int w = 0; w < p.runs; ++w) m = fmaxf(m, red_ml[w * p.row_waves + row_wave][16 * rb + li].x);
        const float ms = m == -INFINITY ? 0.f : m;
        float l = 0.f;
        for (int w = 0; w < p.runs; ++w) {
            const float2 x = red_ml[w * p.row_waves + row_wave][16 * rb + li];
            l += x.y * __builtin_amdgcn_exp2f(x.x - ms);
        }
        const float inv = l > 0.f ? 1.f / l : l;     // (a sum that is not a number stays one)
        if (run == 0 && lg == 0) ml[16 * rb + li] = make_float2(m, trow[rb] >= 0 ? l : 0.f);
        for (int db = run; db < 8; db += p.runs) {
            f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < p.runs; ++w) {
                const int from = w * p.row_waves + row_wave;
                o += red[(from * 8 + db) * kWave + lane] * __builtin_amdgcn_exp2f(red_ml[from][16 * rb + li].x - ms);
            }
            o *= inv;
            if (p.direct_out) {
                if (trow[rb] >= 0) {
                    uint16_t* op = static_cast<uint16_t*>(a.out) + q_first + (int64_t)qrow[rb] * kD + 16 * db + 4 * lg;
                    *reinterpret_cast<uint2*>(op) = make_uint2(Mma<DT>::pack(o[0], o[1]), Mma<DT>::pack(o[2], o[3]));
                }
            } else {
                *reinterpret_cast<f32x4*>(opart + (16 * rb + li) * kD + 16 * db + 4 * lg) = o;
            }
        }
    };
    meet(std::integral_constant<int, 0>{});
    if constexpr (NRB > 1) meet(std::integral_constant<int, 1>{});
}

// Merges the splits' partial rows: half a wavefront per row, four channels per lane.
template <int DT>
__global__ __launch_bounds__(256) void q4_combine_kernel(AttnArgs a, Plan p) {
    const int b = blockIdx.z, unit = b * p.units_per_b + (int)blockIdx.y;
    const int hkv = (int)div_exact(blockIdx.y, (unsigned)p.n_rg), rg = (int)blockIdx.y - hkv * p.n_rg;
    const int row = (int)blockIdx.x * 8 + (int)threadIdx.x / 32, c = 4 * (threadIdx.x & 31);
    const int tq = max(min(a.q_off[b + 1] - a.q_off[b], a.max_tq), 0);
    const int m2 = rg * p.rows_wg + row;
    if (row >= p.rows_wg || m2 >= p.group * tq) return;
    const char* ws = static_cast<const char*>(a.workspace);
    const int64_t first = (int64_t)unit * p.nsplit * p.rows_wg + row;
    const float2* ml = reinterpret_cast<const float2*>(ws + p.off_ml) + first;
    const float* opart = reinterpret_cast<const float*>(ws + p.off_opart) + first * kD + c;
    float m = -INFINITY;
    for (int s = 0; s < p.nsplit; ++s) m = fmaxf(m, ml[(int64_t)s * p.rows_wg].x);
    m = m == -INFINITY ? 0.f : m;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
    for (int s = 0; s < p.nsplit; ++s) {
        const float2 x = ml[(int64_t)s * p.rows_wg];
        const float w = x.y * __builtin_amdgcn_exp2f(x.x - m);
        l += w;
        o += *reinterpret_cast<const f32x4*>(opart + (int64_t)s * p.rows_wg * kD) * w;
    }
    o *= l > 0.f ? 1.f / l : l;
    const int t = (int)div_exact((unsigned)m2, (unsigned)p.group), g = m2 - t * p.group;
    uint16_t* op = static_cast<uint16_t*>(a.out) + (((int64_t)a.q_off[b] + t) * a.n_q_heads + hkv * p.group + g) * kD + c;
    *reinterpret_cast<uint2*>(op) = make_uint2(Mma<DT>::pack(o[0], o[1]), Mma<DT>::pack(o[2], o[3]));
}

// Per (unit, slot): sum over the unit's rows of sum * exp2(max - row max) / row sum.  Slots that no run wrote hold anything and are not read later.
__global__ __launch_bounds__(256) void q4_slots_kernel(AttnArgs a, Plan p) {
    __shared__ float2 stat[16 * 2 * kWaves];         // (row max, 1 / row sum)
    const int unit = blockIdx.x;
    const int b = (int)div_exact((unsigned)unit, (unsigned)p.units_per_b);
    const int rg = (unit - b * p.units_per_b) % p.n_rg;
    const int tq = max(min(a.q_off[b + 1] - a.q_off[b], a.max_tq), 0);
    const int rows = min(p.rows_wg, p.group * tq - rg * p.rows_wg);
    char* ws = static_cast<char*>(a.workspace);
    const float2* ml = reinterpret_cast<const float2*>(ws + p.off_ml) + (int64_t)unit * p.nsplit * p.rows_wg;
    for (int row = threadIdx.x; row < rows; row += 256) {
        float m = -INFINITY, l = 0.f;
        for (int s = 0; s < p.nsplit; ++s) m = fmaxf(m, ml[s * p.rows_wg + row].x);
        m = m == -INFINITY ? 0.f : m;
        for (int s = 0; s < p.nsplit; ++s) l += ml[s * p.rows_wg + row].y * __builtin_amdgcn_exp2f(ml[s * p.rows_wg + row].x - m);
        stat[row] = make_float2(m, l > 0.f ? 1.f / l : l);
    }
    __syncthreads();
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const float2* massml = reinterpret_cast<const float2*>(ws + p.off_massml) + (int64_t)unit * p.slots * p.rows_wg;
    float* masspart = reinterpret_cast<float*>(ws + p.off_masspart) + (int64_t)unit * p.slots;
    for (int k = wave; k < p.slots; k += 4) {
        float c = 0.f;
        for (int row = lane; row < rows; row += kWave) {
            const float2 v = massml[(int64_t)k * p.rows_wg + row];
            c += v.y * __builtin_amdgcn_exp2f(v.x - stat[row].x) * stat[row].y;
        }
        c = wave_sum(c);
        if (lane == 0) masspart[k] = c;
    }
}

// Per-segment attention mass of one query, then S += mass (Alg. 2): sums over units, then over the runs that hold the segment's tiles, in
// a fixed order; a document slot's first entry adds up all of the slot's entries.
__global__ __launch_bounds__(256) void q4_mass_kernel(AttnArgs a, Plan p) {
    __shared__ SegTable tbl;
    __shared__ float col[kMaxEntries + kMaxSplit * kWaves], seg_mass[kMaxEntries];
    const int b = blockIdx.x, tid = threadIdx.x;
    const QueryHead qh = load_query_head(a, b, tid);
    build_table(a, qh, &tbl, kTile);
    const float* part = reinterpret_cast<const float*>(static_cast<const char*>(a.workspace) + p.off_masspart) + (int64_t)b * p.units_per_b * p.slots;
    for (int k = tid; k < p.slots; k += 256) {
        float c = 0.f;
        for (int u = 0; u < p.units_per_b; ++u) c += part[(int64_t)u * p.slots + k];
        col[k] = c;
    }
    __syncthreads();
    const int total = tbl.tile0[tbl.n], nsub = p.nsplit * p.runs;
    if (tid < tbl.n) {
        const int ts = tbl.tile0[tid], te = tbl.tile0[tid + 1];
        float m = 0.f;
        if (te > ts) {
            for (int sub = (int)((((int64_t)ts + 1) * nsub - 1) / total); sub < nsub; ++sub) {
                const int r0 = run_begin(total, nsub, sub), r1 = run_begin(total, nsub, sub + 1);
                if (r0 >= te) break;
                if (r1 > r0 && r1 > ts) m += col[tid + sub];
            }
        }
        a.mass[(int64_t)b * a.seg_stride + tid] = m;
        seg_mass[tid] = m;
    }
    __syncthreads();
    if (a.score_accum == nullptr || tid >= tbl.n) return;
    const int d = tbl.doc[tid];
    if (d < 0 || d >= a.score_stride) return;
    float sum = seg_mass[tid];
    for (int j = 0; j < tbl.n; ++j) {
        if (tbl.doc[j] != d) continue;
        if (j < tid) return;
        if (j > tid) sum += seg_mass[j];
    }
    a.score_accum[(int64_t)b * a.score_stride + d] += sum;
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
    const dim3 grid((unsigned)p.nsplit, (unsigned)p.units_per_b, (unsigned)a.batch), block(kThreads);
    auto go = [&](auto dt, auto pairing, auto nrb) {
        constexpr int DT = decltype(dt)::value, PAIRING = decltype(pairing)::value, NRB = decltype(nrb)::value;
        // (with two row blocks a wavefront has no registers left for a table)
        if constexpr (NRB == 1) {
            if (a.seg_stride <= kWave) {
                hipLaunchKernelGGL((attn_q4_kernel<DT, PAIRING, 1, true>), grid, block, 0, s, a, f, p, sc);
                return;
            }
        }
        hipLaunchKernelGGL((attn_q4_kernel<DT, PAIRING, NRB, false>), grid, block, 0, s, a, f, p, sc);
    };
    auto by_rows = [&](auto dt, auto pairing) {
        if (p.nrb == 1) go(dt, pairing, std::integral_constant<int, 1>{});
        else go(dt, pairing, std::integral_constant<int, 2>{});
    };
    auto by_pairing = [&](auto dt) {
        if (a.pairing == CF_ROPE_HALF) by_rows(dt, std::integral_constant<int, CF_ROPE_HALF>{});
        else by_rows(dt, std::integral_constant<int, CF_ROPE_INTERLEAVED>{});
    };
    const bool bf16 = a.dtype == CF_BF16;
    if (bf16) by_pairing(std::integral_constant<int, CF_BF16>{});
    else by_pairing(std::integral_constant<int, CF_F16>{});
    CF_HIP(hipGetLastError());
    if (!p.direct_out) {
        const dim3 rows((unsigned)(p.rows_wg + 7) / 8, (unsigned)p.units_per_b, (unsigned)a.batch);
        if (bf16) hipLaunchKernelGGL(q4_combine_kernel<CF_BF16>, rows, dim3(256), 0, s, a, p);
        else hipLaunchKernelGGL(q4_combine_kernel<CF_F16>, rows, dim3(256), 0, s, a, p);
        CF_HIP(hipGetLastError());
    }
    if (a.mass != nullptr) {
        hipLaunchKernelGGL(q4_slots_kernel, dim3((unsigned)p.units), dim3(256), 0, s, a, p);
        hipLaunchKernelGGL(q4_mass_kernel, dim3((unsigned)a.batch), dim3(256), 0, s, a, p);
        CF_HIP(hipGetLastError());
    }
    return CF_OK;
}

}  // namespace cf
