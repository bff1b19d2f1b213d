// The writer of the cache store in 4 bits: fresh keys, turned to the position they are cached at (Eq. 5), and values go to their slots
// as four-bit codes with a scale byte per 32 channels.  One pass, bound by HBM: 512 bytes of a key and a value row in, 136 out (4800 tokens of
// 32 heads: 23.4 us = 4.3 TB/s, 87 % of what a 2 GiB copy reaches; 64 tokens of 4 heads 4.3 us, a launch's latency).
#include "cf_common.h"

namespace cf {
namespace {

constexpr int kThreads = 256;
constexpr int kLanes = 8;                            // lanes of a row: 8 + 8 of its 128 channels each
constexpr int kRows = kThreads / kLanes;             // (token, kv head) rows of a workgroup
constexpr int kSlices = 64;

// The scale byte of a group whose largest magnitude has the bits `top`: the smallest power of two with magnitude <= 7 * scale — so the largest
// value is at most half a step from a code — within exponents [lo, hi]; 255 if a value is not finite.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top, int lo, int hi) {
    if (top >= 0x7f800000u) return 255;
    const int e = (int)(top >> 23) - 127 - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);      // (below fp32's normal numbers: under lo anyway)
    return (uint32_t)(127 + min(max(e, lo), hi));
}

// Eight values as codes (nearest, ties to the even index, past 6 to 6).
__device__ __forceinline__ uint32_t codes8(const float (&v)[8], uint32_t byte) {
    if (byte == 255) return 0;
    const float scale = __uint_as_float(byte << 23);
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
}

// the largest magnitude as the bits of a float (so that a NaN counts as the largest): of eight values, and over `lanes` neighbouring lanes
__device__ __forceinline__ uint32_t top_of(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
}
__device__ __forceinline__ uint32_t top_across(uint32_t m, int lanes) {
    for (int o = 1; o < lanes; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    return m;
}

template <int DT>
__device__ __forceinline__ void load8(const void* base, int64_t at, float (&v)[8]) {
    const uint4 w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = DT == CF_BF16 ? bf16_bits_to_float(u[i] & 0xffffu) : f16_bits_to_float(u[i] & 0xffffu);
        v[2 * i + 1] = DT == CF_BF16 ? bf16_bits_to_float(u[i] >> 16) : f16_bits_to_float(u[i] >> 16);
    }
}

// Row r is kv head r % heads of token r / heads.  A lane has two runs of eight channels: [8j, 8j + 8) and 64 further on with half-split
// pairs, [16j, 16j + 16) with interleaved ones, so that both channels of a slice are its own; 32 channels of a scale are those of four
// lanes (half-split) or two.
// Keys are turned in fp64 and rounded to fp32: next to a border between two codes an fp32 rotation would pick another code than the
// definition, a difference of half the value.  (The turn costs less than the memory pass: its angles are worked out once per token.)
template <int DT, int PAIRING>
__global__ __launch_bounds__(kThreads) void quantize_kernel(QuantizeArgs a, RopeFreq freq) {
    __shared__ double2 cs[(kRows + 1) * kSlices];
    const int tid = threadIdx.x, j = tid & (kLanes - 1);
    const int64_t row0 = (int64_t)blockIdx.x * kRows, n_rows = (int64_t)a.n_tokens * a.n_kv_heads;
    const int64_t row = min(row0 + tid / kLanes, n_rows - 1);
    const int tok = (int)(row / a.n_kv_heads), head = (int)(row - (int64_t)tok * a.n_kv_heads);
    const int tok_first = (int)(row0 / a.n_kv_heads);
    const int o0 = PAIRING == CF_ROPE_HALF ? 8 * j : 16 * j, o1 = PAIRING == CF_ROPE_HALF ? kSlices + 8 * j : 16 * j + 8;
    const int64_t src = row * (2 * kSlices);
    float k0[8], k1[8], v0[8], v1[8];
    load8<DT>(a.k, src + o0, k0);
    load8<DT>(a.k, src + o1, k1);
    load8<DT>(a.v, src + o0, v0);
    load8<DT>(a.v, src + o1, v1);
    const int64_t slot = a.n_live && tok >= *a.n_live ? -1 : a.slots[tok];
    const int shift = a.shift ? a.shift[tok] : 0;
    if (a.shift) {
        // tokens of the workgroup's rows, from row numbers counted from its first token's (which 32 bits hold)
        const int n_tok = (int)(min(row0 + kRows, n_rows) - 1 - (int64_t)tok_first * a.n_kv_heads) / a.n_kv_heads + 1;
        for (int i = tid; i < n_tok * kSlices; i += kThreads) {
            const double x = (double)a.shift[tok_first + i / kSlices] * freq.rev[i % kSlices];
            double s, c;
            sincospi(2.0 * (x - rint(x)), &s, &c);
            cs[i] = make_double2(c, s);
        }
        __syncthreads();
    }
    const bool off_range = shift <= -a.max_positions || shift >= a.max_positions;
    const bool live = row0 + tid / kLanes < n_rows && slot >= 0 && slot < a.n_store_tokens && !off_range;
    if (row0 + tid / kLanes < n_rows && j == 0 && head == 0 && slot >= 0) {
        if (slot >= a.n_store_tokens) raise_flag(a.dev_flag, CF_FLAG_BAD_INDEX);
        else if (off_range) raise_flag(a.dev_flag, CF_FLAG_POS_RANGE);
    }
    if (shift != 0) {
        const double2* w = cs + (tok - tok_first) * kSlices;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (PAIRING == CF_ROPE_HALF) {
                const double2 c = w[8 * j + i];
                const double x = k0[i], y = k1[i];
                k0[i] = (float)(x * c.x - y * c.y);
                k1[i] = (float)(x * c.y + y * c.x);
            } else {
                const double2 c = w[8 * j + i];
                float* p = i < 4 ? k0 + 2 * i : k1 + 2 * (i - 4);
                const double x = p[0], y = p[1];
                p[0] = (float)(x * c.x - y * c.y);
                p[1] = (float)(x * c.y + y * c.x);
            }
        }
    }
    uint32_t byte[4];                                // of k0, k1, v0, v1
    if (PAIRING == CF_ROPE_HALF) {
        byte[0] = scale_byte(top_across(top_of(k0), 4), a.e_lo, a.e_hi);
        byte[1] = scale_byte(top_across(top_of(k1), 4), a.e_lo, a.e_hi);
        byte[2] = scale_byte(top_across(top_of(v0), 4), a.e_lo, a.e_hi);
        byte[3] = scale_byte(top_across(top_of(v1), 4), a.e_lo, a.e_hi);
    } else {
        byte[0] = byte[1] = scale_byte(top_across(max(top_of(k0), top_of(k1)), 2), a.e_lo, a.e_hi);
        byte[2] = byte[3] = scale_byte(top_across(max(top_of(v0), top_of(v1)), 2), a.e_lo, a.e_hi);
    }
    if (!live) return;
    const int64_t at = slot * a.store_ts + (int64_t)head * a.store_hs;
    uint32_t* kc = reinterpret_cast<uint32_t*>(a.k_codes + (at >> 1));
    uint32_t* vc = reinterpret_cast<uint32_t*>(a.v_codes + (at >> 1));
    kc[o0 >> 3] = codes8(k0, byte[0]);
    kc[o1 >> 3] = codes8(k1, byte[1]);
    vc[o0 >> 3] = codes8(v0, byte[2]);
    vc[o1 >> 3] = codes8(v1, byte[3]);
    if (PAIRING == CF_ROPE_HALF ? (j & 3) == 0 : (j & 1) == 0) {
        const int g0 = o0 / 32, g1 = o1 / 32;
        a.k_scales[(at >> 5) + g0] = (uint8_t)byte[0];
        a.v_scales[(at >> 5) + g0] = (uint8_t)byte[2];
        if (PAIRING == CF_ROPE_HALF) {
            a.k_scales[(at >> 5) + g1] = (uint8_t)byte[1];
            a.v_scales[(at >> 5) + g1] = (uint8_t)byte[3];
        }
        if (byte[0] == 255 || byte[1] == 255 || byte[2] == 255 || byte[3] == 255) raise_flag(a.dev_flag, CF_FLAG_NONFINITE_VALUE);
    }
}

}  // namespace

cf_status launch_quantize(const cf_layer_desc* d, const RopeFreq& f, QuantizeArgs a, hipStream_t s) {
    // exponents at which every code is a number of the 16-bit type (bf16: a normal one)
    a.e_lo = d->dtype == CF_BF16 ? -125 : -23;
    a.e_hi = d->dtype == CF_BF16 ? 125 : 13;
    const int64_t blocks = ((int64_t)a.n_tokens * a.n_kv_heads + kRows - 1) / kRows;
    CF_REQUIRE(blocks <= 0x7fffffff, CF_ERR_UNSUPPORTED, "n_tokens * n_kv_heads too large");
    auto go = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (d->rope_pairing == CF_ROPE_HALF)
            hipLaunchKernelGGL((quantize_kernel<DT, CF_ROPE_HALF>), dim3((unsigned)blocks), dim3(kThreads), 0, s, a, f);
        else
            hipLaunchKernelGGL((quantize_kernel<DT, CF_ROPE_INTERLEAVED>), dim3((unsigned)blocks), dim3(kThreads), 0, s, a, f);
    };
    if (d->dtype == CF_BF16) go(std::integral_constant<int, CF_BF16>{});
    else go(std::integral_constant<int, CF_F16>{});
    CF_HIP(hipGetLastError());
    return CF_OK;
}

}  // namespace cf
