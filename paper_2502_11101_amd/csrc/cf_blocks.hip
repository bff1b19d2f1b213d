// One scheduler step of a cache kept in blocks: from the requests' lengths the blocks they get and give back, the slots of their new tokens
// and the segment tables and row offsets that the attention takes.  Integer work on a few KB per request, bound by latency: one
// launch, a workgroup per request, each of which adds up the requests ahead of its own by itself (one request 4.7 us, 512 of them 9.7).
#include "cf_common.h"

namespace cf {
namespace {

constexpr int kThreads = 256;
constexpr int kWavesHere = kThreads / kWave;

// x / block_tokens for 0 <= x < 2^33: the estimate is off by at most one (a tenth of the instructions of a 64-bit division)
struct Blocks {
    int64_t tokens;
    double per_token;
    __device__ __forceinline__ explicit Blocks(int32_t block_tokens) : tokens(block_tokens), per_token(1.0 / block_tokens) {}
    __device__ __forceinline__ int64_t of(int64_t x) const {
        int64_t q = (int64_t)((double)x * per_token);
        const int64_t r = x - q * tokens;
        q += (r >= tokens ? 1 : 0) - (r < 0 ? 1 : 0);
        return q;
    }
    __device__ __forceinline__ int64_t up(int64_t x) const { return of(x + tokens - 1); }
};

// What a request asks for.
struct Ask {
    int64_t rows;       // new tokens
    int64_t want;       // blocks it needs beyond those it holds
    int64_t have;       // blocks it holds
    bool leaves, bad;   // gives its blocks back; its lengths do not fit its table, or its rows the step
    bool lost;          // not even what it holds is known
    bool over;          // more rows than a request may have, or than the step has room for
};
// `fit`: the requests ahead of this one have room for all their rows.
__device__ __forceinline__ Ask ask_of(const BlockArgs& a, const Blocks& blocks, int i, int fit) {
    const int64_t cached = a.cached[i], fresh = a.fresh[i];
    Ask k;
    k.leaves = fresh < 0;
    k.rows = k.leaves ? 0 : fresh;
    k.have = blocks.up(max(cached, (int64_t)0));
    const int64_t need = blocks.up(max(cached, (int64_t)0) + k.rows);
    k.over = k.rows > 0 && (i >= fit || (a.max_fresh > 0 && k.rows > a.max_fresh));
    k.bad = cached < 0 || k.have > a.table_stride || (!k.leaves && need > a.table_stride) || k.over;
    k.lost = cached < 0 || k.have > a.table_stride;
    if (k.lost) k.have = 0;
    k.want = k.leaves || k.bad ? 0 : need - k.have;
    return k;
}

__device__ __forceinline__ int64_t wave_sum64(int64_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
// sums of N values over the workgroup, in every thread
template <int N> __device__ __forceinline__ void block_sums(int64_t (&v)[N], int64_t (*lds)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum64(v[i]);
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) lds[threadIdx.x / kWave][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = 0;
        for (int w = 0; w < kWavesHere; ++w) v[i] += lds[w][i];
    }
}
// inclusive prefix sum over the workgroup's threads
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* lds) {
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const int64_t u = __shfl_up(v, o);
        if (lane >= o) v += u;
    }
    __syncthreads();
    if (lane == kWave - 1) lds[wave] = v;
    __syncthreads();
    for (int w = 0; w < wave; ++w) v += lds[w];
    return v;
}

// how many threads up to this one, it included, have their flag set
__device__ __forceinline__ int64_t block_count(bool flag, int64_t* lds) {
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const uint64_t all = __ballot(flag);
    int64_t v = __popcll(all & (~0ull >> (kWave - 1 - lane)));
    __syncthreads();
    if (lane == 0) lds[wave] = __popcll(all);
    __syncthreads();
    for (int w = 0; w < wave; ++w) v += lds[w];
    return v;
}

// dynamic LDS: the request's blocks [table_stride], starts of its runs [table_stride + 1], and, where requests leave, how many blocks those up
// to each give back [batch]
__global__ __launch_bounds__(kThreads) void block_tables_kernel(BlockArgs a) {
    extern __shared__ int32_t smem[];
    __shared__ int64_t sums[kWavesHere][4], scan[kWavesHere];
    int32_t* const ids = smem;
    int32_t* const starts = ids + a.table_stride;
    int32_t* const back_upto = starts + a.table_stride + 1;
    const int b = blockIdx.x, tid = threadIdx.x;
    const Blocks blocks(a.block_tokens);

    // ---- the requests ahead of this one, and all of them
    // (wants and returns of all requests are less than 2^31, kMaxBlockBatch times kMaxBlockTable: two counts to a sum)
    int64_t t[4];                                    // rows, wants and returns ahead; rows, wants and returns of all
    auto tally = [&](int fit) {
        for (int j = 0; j < 4; ++j) t[j] = 0;
        for (int i = tid; i < a.batch; i += kThreads) {
            const Ask k = ask_of(a, blocks, i, fit);
            const int64_t blocks_of = k.want | (k.leaves ? k.have : 0) << 32;
            if (i < b) { t[0] += k.rows; t[1] += blocks_of; }
            t[2] += k.rows;
            t[3] += blocks_of;
        }
        block_sums<4>(t, sums);
    };
    int fit = a.batch;
    tally(fit);
    if (a.max_fresh > 0 && t[2] > a.max_new_tokens) {                // workgroup-uniform: the requests up to the first whose rows run past the room
        int64_t carry = 0;
        fit = 0;
        for (int i0 = 0; i0 < a.batch; i0 += kThreads) {
            const int i = i0 + tid;
            const int64_t upto = carry + block_scan(i < a.batch ? ask_of(a, blocks, i, a.batch).rows : 0, scan);
            fit += __syncthreads_count(i < a.batch && upto <= a.max_new_tokens);
            if (tid == kThreads - 1) scan[0] = upto;
            __syncthreads();
            carry = scan[0];
        }
        tally(fit);
    }
    const int64_t rows_before = t[0], want_before = (uint32_t)t[1], back_before = t[1] >> 32, back_all = t[3] >> 32;
    const Ask me = ask_of(a, blocks, b, fit);
    const int64_t n_free_raw = a.n_free[0];
    const int64_t n_free = min(max(n_free_raw, (int64_t)0), (int64_t)a.n_blocks);
    const int64_t room = n_free + back_all;          // what the free list holds before anything is taken off it
    // what is handed out: all of it, or where the list runs short the wants of the requests that still fit
    int64_t granted = (uint32_t)t[3];
    if (granted > room) {
        int64_t carry = 0;
        granted = 0;
        for (int i0 = 0; i0 < a.batch; i0 += kThreads) {
            const int i = i0 + tid;
            const int64_t upto = carry + block_scan(i < a.batch ? ask_of(a, blocks, i, fit).want : 0, scan);
            int64_t most[1] = {upto <= room ? upto : 0};
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) most[0] = max(most[0], (int64_t)__shfl_xor(most[0], o));
            __syncthreads();
            if ((tid & (kWave - 1)) == 0) scan[tid / kWave] = most[0];
            __syncthreads();
            for (int w = 0; w < kWavesHere; ++w) granted = max(granted, scan[w]);
            __syncthreads();
            if (tid == kThreads - 1) scan[0] = upto;
            __syncthreads();
            carry = scan[0];
        }
    }
    const int64_t left = room - granted;
    const bool served = !me.bad && (me.want == 0 || want_before + me.want <= room);
    if (back_all > 0) {                              // workgroup-uniform
        int64_t carry = 0;
        for (int i0 = 0; i0 < a.batch; i0 += kThreads) {
            const int i = i0 + tid;
            int64_t mine = 0;
            if (i < a.batch) {
                const Ask k = ask_of(a, blocks, i, fit);
                mine = k.leaves ? k.have : 0;
            }
            const int64_t upto = carry + block_scan(mine, scan);
            if (i < a.batch) back_upto[i] = (int32_t)min(upto, (int64_t)0x7fffffff);
            __syncthreads();
            if (tid == kThreads - 1) scan[0] = upto;
            __syncthreads();
            carry = scan[0];
            __syncthreads();
        }
    }

    // ---- blocks: those held, and new ones off the top of the free list
    bool off_table = false;
    for (int j = tid; j < me.have; j += kThreads) ids[j] = a.table[(int64_t)b * a.table_stride + j];
    if (served)
        for (int i = tid; i < me.want; i += kThreads) {
            const int64_t at = room - 1 - (want_before + i);
            int32_t id = -1;
            if (at < n_free) {
                id = a.free_blocks[at];
            } else {                                 // one that a request gives back in this step
                const int r = (int)(at - n_free);
                int lo = 0, hi = a.batch - 1;        // the first request whose returns reach past r
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (back_upto[mid] > r) hi = mid;
                    else lo = mid + 1;
                }
                id = a.table[(int64_t)lo * a.table_stride + r - (lo ? back_upto[lo - 1] : 0)];
            }
            off_table |= id < 0 || id >= a.n_blocks;
            ids[me.have + i] = id;
            a.table[(int64_t)b * a.table_stride + me.have + i] = id;
        }
    __syncthreads();
    const int64_t cached = a.cached[b];
    const bool lost = me.lost;
    if (me.leaves)                                   // its blocks go on top of the free list, below what is handed on
        for (int j = tid; j < me.have; j += kThreads) {
            const int64_t at = n_free + back_before + j;
            if (at < left && at < a.n_blocks) a.free_blocks[at] = ids[j];
            off_table |= at >= a.n_blocks || ids[j] < 0 || ids[j] >= a.n_blocks;
        }

    // ---- rows, positions, slots
    const int64_t position = a.position ? a.position[b] : 0;
    const int64_t q_new = min(position + (me.leaves || lost ? 0 : cached), (int64_t)0x7fffffff);
    bool too_many = false;
    for (int64_t r = tid; r < me.rows; r += kThreads) {
        const int64_t at = rows_before + r;
        if (at >= a.max_new_tokens) { too_many = true; break; }
        int64_t slot = -1;
        if (served) {
            const int64_t tok = cached + r, j = blocks.of(tok);
            const int32_t id = ids[j];
            if (id >= 0 && id < a.n_blocks) slot = a.first_token + (int64_t)id * a.block_tokens + (tok - j * a.block_tokens);
            else off_table = true;
        }
        a.slots[at] = slot;
        a.shift[at] = (int32_t)(q_new - a.q_stored_start);
    }

    // ---- the segment table: shared entries, runs of neighbouring blocks, the own rows
    int n_base = 0;
    bool bad_base = false;
    if (a.n_base && !me.leaves && !lost && !me.over) {
        n_base = a.n_base[b];
        bad_base = n_base < 0 || n_base > a.base_stride;
        n_base = min(max(n_base, 0), a.base_stride);
    }
    int n_run = 0;
    if (!me.leaves && !me.over) {
        int64_t carry = 0;
        for (int64_t j0 = 0; j0 < me.have; j0 += kThreads) {
            const int64_t j = j0 + tid;
            const bool starts_run = j < me.have && (j == 0 || ids[j] != ids[j - 1] + 1);
            const int64_t upto = carry + block_count(starts_run, scan);
            if (starts_run) starts[upto - 1] = (int32_t)j;
            __syncthreads();
            if (tid == kThreads - 1) scan[0] = upto;
            __syncthreads();
            carry = scan[0];
            __syncthreads();
        }
        n_run = (int)carry;
        if (tid == 0) starts[n_run] = (int32_t)me.have;
    }
    __syncthreads();
    const bool own = me.rows > 0 && !lost && !me.over;
    const int n = n_base + n_run + (own ? 1 : 0);
    const bool fits = n <= a.seg_stride;
    cf_segment* const out = a.segs + (int64_t)b * a.seg_stride;
    if (fits) {
        for (int i = tid; i < n_base; i += kThreads) out[i] = a.base_segs[(int64_t)b * a.base_stride + i];
        for (int i = tid; i < n_run; i += kThreads) {
            const int j0 = starts[i], j1 = starts[i + 1];
            const int64_t tok = (int64_t)j0 * a.block_tokens;
            const int32_t id = ids[j0];
            const bool ok = id >= 0 && (int64_t)id + (j1 - j0) <= a.n_blocks;
            off_table |= !ok;
            cf_segment s;
            s.tok_offset = ok ? a.first_token + (int64_t)id * a.block_tokens : 0;
            s.len = ok ? (int32_t)(min((int64_t)j1 * a.block_tokens, cached) - tok) : 0;
            s.stored_start = s.new_start = (int32_t)min(position + tok, (int64_t)0x7fffffff);
            s.kind = CF_SEG_PREFIX;
            s.doc = -1;
            s.reserved = 0;
            out[n_base + i] = s;
        }
        if (own && tid == 0) {
            cf_segment s;
            s.tok_offset = rows_before;
            s.len = (int32_t)me.rows;
            s.stored_start = a.q_stored_start;
            s.new_start = (int32_t)q_new;
            s.kind = CF_SEG_SELF;
            s.doc = -1;
            s.reserved = 0;
            out[n - 1] = s;
        }
    }
    if (off_table || too_many || ((me.bad || n_free_raw != n_free) && tid == 0)) raise_flag(a.dev_flag, CF_FLAG_BAD_INDEX);
    if (tid != 0) return;
    if (!served && !me.bad) raise_flag(a.dev_flag, CF_FLAG_NO_BLOCKS);
    if (!fits || bad_base) raise_flag(a.dev_flag, CF_FLAG_BAD_SEGMENT);
    a.n_seg[b] = fits ? n : 0;
    a.next_len[b] = me.leaves ? 0 : (int32_t)(served ? cached + me.rows : cached);
    a.q_new_start[b] = (int32_t)q_new;
    const int64_t most = a.max_fresh > 0 ? min(a.max_new_tokens, (int64_t)0x7fffffff) : 0x7fffffff;
    if (b == 0) { a.q_off[0] = 0; a.next_n_free[0] = (int32_t)min(left, (int64_t)a.n_blocks); }
    a.q_off[b + 1] = (int32_t)min(rows_before + me.rows, most);
    if (rows_before + me.rows > most) raise_flag(a.dev_flag, CF_FLAG_BAD_INDEX);
}

}  // namespace

cf_status launch_block_tables(const BlockArgs& a, hipStream_t s) {
    const size_t lds = ((size_t)2 * a.table_stride + 1 + a.batch) * sizeof(int32_t);
    hipLaunchKernelGGL(block_tables_kernel, dim3((unsigned)a.batch), dim3(kThreads), lds, s, a);
    CF_HIP(hipGetLastError());
    return CF_OK;
}

}  // namespace cf
