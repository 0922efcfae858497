// sbw_token_logprobs and sbw_token_logprobs_backward: log probabilities of given tokens with the
// entropy of their rows, their ranks and the most probable alternatives, under the softmax of the
// logits or of the watermarked logits (Eq. 1 and Eq. 2 applied on the way), and the gradient of
// log probability and entropy with respect to the logits.
//
// Mathematics.  With l the (biased) logits of a row, c = log2(e) / tau and a reference m, a thread
// keeps Z = sum 2^((l-m)c) and S = sum 2^((l-m)c) (l-m)c over its columns; moving the reference
// from m to m' by d = (m-m')c turns (Z, S) into (2^d Z, 2^d (S + d Z)).  One pass over the row and a
// merge then give
//     log p_v = (l_v - m)/tau - ln Z            H = ln Z - ln 2 * S/Z.
// The gradient needs no reduction at all: with the saved m, Z and H,
//     dl_v = 1/tau [ g (1[v = t] - p_v) - h p_v (ln p_v + H) ].
//
// What bounds them (B200, device time in graph replay).  Plain logits: memory -- 4096 x 128256 bf16 are
// read in 181 to 190 us, by the clock that the power cap leaves, 5.5 to 5.8 TB/s or 84 to 89 % of the measured copy rate; with the
// exponentials taken out the same loads run at that rate, with them the SFU is busy 66 % and the issue slots 62 % of the
// time (8 instructions a logit, one an exponential).  Watermarked logits: the 32x32->64 multiplies of the hash --
// 592 x 128256 bf16 380 Gelem/s, 592 x 151936 fp32 self-salt 221 Gelem/s, 0.75 to 0.8 of what the bias kernel reaches; 64
// rows on 148 SMs lose another seventh to whole CTAs.
// A handful of rows: latency -- one row of 128256 with 20 alternatives 8.6 us, of which the last 4.4 us are the
// short dependent phases after the row's last byte (bound, hits, second look, ranking, merge).  The gradient:
// memory -- 2048 x 128256 bf16 in 160 us, the measured copy rate; watermarked 345 Gelem/s, self-salt 230 to 238.
#include <cooperative_groups.h>

#include <atomic>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "sbw_codes.cuh"
#include "sbw_common.cuh"
#include "sbw_rowbias.cuh"

namespace sbw {
namespace {

// CTA size.  Without the hash three CTAs of 256 threads per SM (80 registers; 4096 x 128256 bf16: 193 us, four at
// 64 registers 202, two of 384 threads 206, one of 512 219).  With it (128 registers) four of 128: the same 16
// warps as the other hashing kernels, in smaller pieces, so that a call's CTAs share the SMs out more
// evenly (64 x 128256 watermarked: 34 us, two of 256 threads 43).
__host__ __device__ constexpr int threads_of(int scheme) { return scheme < 0 ? 256 : 128; }
__host__ __device__ constexpr int ctas_per_sm(int scheme) { return scheme < 0 ? 3 : 4; }
constexpr int kCap = 1280;              // candidate list entries
constexpr int kBlocks = 8;              // blocks of trips whose maxima a thread remembers
constexpr int kHits = 512;              // blocks that reach the bound
constexpr int kMaxTop = SBW_MAX_TOP_LOGPROBS;
// CTAs per row at most
__host__ __device__ constexpr int max_parts(bool top) { return top ? 8 : 16; }
constexpr float kFar = -300.0f;         // exponents below this give 2^x = 0; keeps 0 * inf out of the sums
static_assert(kCap >= 16 * kMaxTop + 16, "a share with vectors for fewer groups than alternatives must fit the list");

struct LogprobArgs {
    const void *logits;
    int64_t B, V, ld;
    const int32_t *ctx;
    int W;
    uint32_t vocab_offset;
    BiasParams bias;
    double inv_tau;
    float c;               // log2(e) / tau, rounded
    double c_off;          // ln 2 times the relative error of that rounding
    float huge;            // ordinary values end here; a bf16 value
    const int32_t *tokens; // nullable
    int top_n;
    float *out_logprob, *out_entropy;
    int32_t *out_rank;
    float *out_max, *out_sumexp;
    int32_t *out_top_ids;
    float *out_top_logprobs;
};

// max that keeps a NaN (fmaxf drops it): a NaN logit has to reach the sums
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Whether `bytes` bytes at p lie in row `row` of a [B, V] block (bounds-flag build).
[[maybe_unused]] __device__ __forceinline__ bool in_row(const void *base, int64_t ld, int64_t B, int64_t V, int esize, int64_t row, const void *p,
                                       int bytes) {
    const char *begin = static_cast<const char *>(base) + row * ld * esize;
    const char *q = static_cast<const char *>(p);
    return row >= 0 && row < B && q >= begin && q + bytes <= begin + V * esize;
}

// ---- where a row's aligned vectors are ----
// Columns [0, head) come before the first 16-byte boundary, then nvec vectors, then the tail.
template <int DTYPE>
struct RowLayout {
    static constexpr int ESIZE = DTYPE == SBW_DTYPE_F32 ? 4 : 2;
    static constexpr int VEC = 16 / ESIZE;
    uint32_t head, nvec;
    __device__ __forceinline__ RowLayout(const char *row_ptr, uint32_t V) {
        const uint32_t skip = (static_cast<uint32_t>(16u - (reinterpret_cast<uintptr_t>(row_ptr) & 15u)) & 15u) / ESIZE;
        head = min(skip, V);
        nvec = (V - head) / VEC;
    }
};

// The value the order goes by: NaN counts as -inf, both zeros are one value.
__device__ __forceinline__ uint32_t value_code(float x) {
    return order_code(__float_as_uint(x == x ? x + 0.0f : -INFINITY));
}
__device__ __forceinline__ uint64_t composite(float x, uint32_t col) {
    return (static_cast<uint64_t>(value_code(x)) << 32) | (0xFFFFFFFFu - col);
}
__device__ __forceinline__ float composite_value(uint64_t e) {
    return __uint_as_float(order_decode(static_cast<uint32_t>(e >> 32)));
}

// Running sums of a set of columns.  Exponents are taken as l c - ref in one fused operation, so ref,
// a rounded m c, is itself the reference: nothing depends on how m c was rounded.
struct Stats {
    float ref, z, s;  // reference (log2 units), sum of 2^(l c - ref), of the same times (l c - ref)
    float top;        // largest value, -inf if none
    uint32_t above;   // columns that rank before the token
    // the same sums with reference `to` >= ref
    __device__ __forceinline__ void move(float to) {
        const float d = fmaxf(ref - to, kFar);
        const float f = ex2_approx_ftz(d);
        s = f * fmaf(d, z, s);
        z *= f;
        ref = to;
    }
};
// Columns below m - 300 / c count as that (2^-300 = 0).  A reference is m c rounded, so the largest column's
// exponent is that rounding and not 0: up to 1 for |m c| < 2^25, but 2^(m c - ref) would overflow from 2^31 on
// (masks of -1e10), and S lose its digits before that.  So 2^25 / c is where ordinary values end
// (LogprobArgs::huge): rows whose largest value is not within +-huge are summed again by sum_plainly, and what lies
// below -2 huge -- far below any largest value that counts -- is taken as that, which is also the reference of a
// warp that has met nothing greater.  With temperatures within 1e-6 .. 1e6 nothing overflows then and no
// 0 * inf arises.
constexpr double kOrdinary = 0x1p25;

// A thread's fp32 sums take in kChain trips; then the warp adds them to its sums in fp64, so that no chain of fp32
// additions grows with the row: at most 16 in a trip, one for its two halves, kChain trips, the row's ragged end and
// five across the warp, 39.  (One chain through the row: 2^20 columns with the hash are 1024 trips, and a term that they
// all repeat was lost to 1.5e-5, one of 2^22 columns to 6e-5.)  Rows whose shares end within kChain trips have kernels
// without that step (LONG): it costs their loop 2 % though it is never taken (4096 x 128256 bf16, sixteen trips: 187 us
// without it, 191 with it, in turn on one GPU).
constexpr uint32_t kChain = 16;
struct WarpSums {
    double z, s;      // as in Stats
    float ref;
    __device__ __forceinline__ void add(const Stats &st) {
        const double d = static_cast<double>(ref) - static_cast<double>(st.ref);     // never above 0
        if (d != 0.0) {
            const double f = exp2(d);
            s = f * fma(d, z, s);
            z *= f;
            ref = st.ref;
        }
        z += static_cast<double>(st.z);
        s += static_cast<double>(st.s);
    }
};

// Largest value of a vector, NaN dropped.
template <int DTYPE>
__device__ __forceinline__ float vector_max(const uint4 &w) {
    if constexpr (DTYPE == SBW_DTYPE_F32) {
        return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
    } else {
        const __nv_bfloat162 *e = reinterpret_cast<const __nv_bfloat162 *>(&w);
        const __nv_bfloat162 m = __hmax2(__hmax2(e[0], e[1]), __hmax2(e[2], e[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
}

// The same over n vectors (bf16: two halves at a time to the end).
template <int DTYPE, int N>
__device__ __forceinline__ float largest_of(const uint4 (&w)[N]) {
    if constexpr (DTYPE == SBW_DTYPE_F32) {
        float m = vector_max<DTYPE>(w[0]);
#pragma unroll
        for (int u = 1; u < N; ++u) m = fmaxf(m, vector_max<DTYPE>(w[u]));
        return m;
    } else {
        const __nv_bfloat162 *e = reinterpret_cast<const __nv_bfloat162 *>(w);
        __nv_bfloat162 m = e[0];
#pragma unroll
        for (int i = 1; i < 4 * N; ++i) m = __hmax2(m, e[i]);
        return fmaxf(__low2float(m), __high2float(m));
    }
}

template <int DTYPE>
__device__ __forceinline__ float element(const uint4 &w, int i) {
    const uint32_t *e = reinterpret_cast<const uint32_t *>(&w);
    if constexpr (DTYPE == SBW_DTYPE_F32) return __uint_as_float(e[i]);
    else return __uint_as_float((i & 1) ? e[i >> 1] & 0xffff0000u : e[i >> 1] << 16);
}

__device__ __forceinline__ uint4 load_vector(const uint4 *p) {
    uint4 r;   // read once, not kept in L1; no .nc: the kernel may write over what it has read
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

// The next value below x in the logits' type (x no NaN and not -inf).
template <int DTYPE>
__device__ __forceinline__ float value_below(float x) {
    constexpr uint32_t ulp = DTYPE == SBW_DTYPE_F32 ? 1u : 0x10000u;
    const uint32_t b = __float_as_uint(x);
    return __uint_as_float((b << 1) == 0 ? 0x80000000u + ulp : (b & 0x80000000u) ? b + ulp : b - ulp);
}
__device__ __forceinline__ uint32_t both_halves(float bf16_value) {
    const uint32_t b = __float_as_uint(bf16_value);
    return (b & 0xffff0000u) | (b >> 16);
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// One (biased) logit of a row, widened.
template <int DTYPE, int SCHEME>
__device__ __forceinline__ float logit_at(const LogprobArgs &a, int64_t row, const char *row_ptr, uint32_t col,
                                          const RowSeedS<SCHEME> &rs) {
    [[maybe_unused]] constexpr int ESIZE = RowLayout<DTYPE>::ESIZE;
    if (!SBW_CHECKED(in_row(a.logits, a.ld, a.B, a.V, ESIZE, row, row_ptr + static_cast<size_t>(col) * ESIZE, ESIZE), SBW_SITE_LOGPROB_LOAD))
        return -INFINITY;
    return biased_at<DTYPE, SCHEME>(row_ptr, col, rs, a.vocab_offset + col, a.bias);
}

// ---- the seldom taken passes over the columns [lo, hi) of a row: plain, one column at a time, out of
// line so that the common path's registers do not pay for them ----
template <int DTYPE, int SCHEME>
struct Columns {
    const LogprobArgs &a;
    const int64_t row;
    const char *row_ptr;
    RowSeedS<SCHEME> rs;
    __device__ __forceinline__ Columns(const LogprobArgs &args, int64_t row_index)
        : a(args), row(row_index), row_ptr(static_cast<const char *>(args.logits) + row * args.ld * RowLayout<DTYPE>::ESIZE) {
        rs.init(args.bias.key, args.ctx + row * args.W, args.W);
    }
    __device__ __forceinline__ float operator[](uint32_t col) const {
        return logit_at<DTYPE, SCHEME>(a, row, row_ptr, col, rs);
    }
};

struct RowSums {
    double z, s;      // as in Stats, relative to the row's largest value
};

// The sums of columns [lo, hi) for rows with values of any size, by the whole CTA: the largest value
// first, then differences.  One thread adds up V / blockDim terms here, so they are added in fp64 (in fp32
// 1000 equal terms in a row would be off by as much as 1.5e-5).
template <int DTYPE, int SCHEME>
__device__ __noinline__ RowSums sum_plainly(const LogprobArgs &a, int64_t row, uint32_t lo, uint32_t hi, float top, RowSums *scratch) {
    const Columns<DTYPE, SCHEME> x(a, row);
    RowSums sums = {0.0, 0.0};
    for (uint32_t col = lo + threadIdx.x; col < hi; col += blockDim.x) {
        const float d = max_nan((x[col] - top) * a.c, kFar);
        const double e = ex2_approx_ftz(d);
        sums.z += e;
        sums.s = fma(e, static_cast<double>(d), sums.s);
    }
    for (int d = 16; d > 0; d >>= 1) {
        sums.z += __shfl_xor_sync(0xffffffffu, sums.z, d);
        sums.s += __shfl_xor_sync(0xffffffffu, sums.s, d);
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = sums;
    __syncthreads();
    sums = {0.0, 0.0};
    for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) {
        sums.z += scratch[w].z;
        sums.s += scratch[w].s;
    }
    return sums;
}

// Columns that rank before column t when its value is -inf (or NaN, which counts as that).
template <int DTYPE, int SCHEME>
__device__ __noinline__ uint32_t count_above_nothing(const LogprobArgs &a, int64_t row, uint32_t lo, uint32_t hi, uint32_t t) {
    const Columns<DTYPE, SCHEME> x(a, row);
    uint32_t n = 0;
    for (uint32_t col = lo + threadIdx.x; col < hi; col += blockDim.x) n += (x[col] > -INFINITY || col < t) ? 1u : 0u;
    return n;
}

// Candidates from `floor` on, or strictly above it.
template <int DTYPE, int SCHEME>
__device__ __noinline__ void gather_again(const LogprobArgs &a, int64_t row, uint32_t lo, uint32_t hi, float floor, bool strict,
                                          uint64_t *list, unsigned *count) {
    const Columns<DTYPE, SCHEME> x(a, row);
    for (uint32_t col = lo + threadIdx.x; col < hi; col += blockDim.x) {
        const float v = x[col];
        if (v > floor || (!strict && v == floor)) {
            const unsigned pos = atomicAdd(count, 1u);
            if (pos < static_cast<unsigned>(kCap)) list[pos] = composite(v, col);
        }
    }
}

// The first columns whose value is `floor` into list[from .. to), in column order; warp 0.
template <int DTYPE, int SCHEME>
__device__ __noinline__ void fill_equal(const LogprobArgs &a, int64_t row, uint32_t lo, uint32_t hi, float floor, uint64_t *list,
                                        unsigned from, unsigned to) {
    const Columns<DTYPE, SCHEME> x(a, row);
    const unsigned lane = threadIdx.x;
    for (uint32_t base = lo; base < hi && from < to; base += 32) {
        const uint32_t col = base + lane;
        const float v = col < hi ? x[col] : 0.0f;
        const bool hit = col < hi && value_code(v) == value_code(floor);
        const unsigned hits = __ballot_sync(0xffffffffu, hit);
        const unsigned pos = from + __popc(hits & ((1u << lane) - 1u));
        if (hit && pos < to) list[pos] = composite(v, col);
        from += __popc(hits);
    }
}

// list[0 .. need): `need` rounds of "largest below the last one"; no assumption about the values.
template <int DTYPE, int SCHEME>
__device__ __noinline__ void select_rounds(const LogprobArgs &a, int64_t row, uint32_t lo, uint32_t hi, uint64_t *list, unsigned need,
                                           uint64_t *scratch) {
    const Columns<DTYPE, SCHEME> x(a, row);
    uint64_t last = ~0ull;
    for (unsigned r = 0; r < need; ++r) {
        uint64_t best = 0;
        for (uint32_t col = lo + threadIdx.x; col < hi; col += blockDim.x) {
            const uint64_t e = composite(x[col], col);
            if (e < last && e > best) best = e;
        }
        for (int d = 16; d > 0; d >>= 1) {
            const uint64_t o = __shfl_xor_sync(0xffffffffu, best, d);
            best = o > best ? o : best;
        }
        if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = best;
        __syncthreads();
        for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) best = scratch[w] > best ? scratch[w] : best;
        if (threadIdx.x == 0) list[r] = best;
        last = best;
        __syncthreads();
    }
}

// ---- the row pass ----
// Every thread copies its own vectors into its own slots of shared memory, groups of a few vectors
// some groups ahead (cp.async: no register waits for the data, no barrier, and a thread waits for
// nothing but its own copies), across row boundaries too, so that the loads go on while a row is finished.
// Three groups of four vectors: 96 KB in flight per SM.  (Four groups: no difference; six or eight vectors a
// group in two groups: 205 us where this took 193; loads into registers a trip ahead: 231 us where the ring took
// 224.)
template <int SCHEME>
struct Ring {
    static constexpr int kGroup = SCHEME == kSchemeNone ? 4 : 2;    // vectors of a group; a trip of the loop takes one
    static constexpr int kStages = SCHEME == kSchemeNone ? 3 : 2;
    static constexpr int kThreads = threads_of(SCHEME);
    static constexpr int kGroupBytes = kGroup * kThreads * 16;
    static constexpr int kBytes = kGroupBytes * kStages;
};
// Vector OFFSET (in vectors) from both addresses, which the instruction adds itself.
template <int OFFSET>
__device__ __forceinline__ void copy_async(uint32_t smem, const uint4 *src) {
    asm volatile("cp.async.cg.shared.global [%0 + %2], [%1 + %2], 16;" ::"r"(smem), "l"(src), "n"(OFFSET * 16));
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N));
}
template <int OFFSET>
__device__ __forceinline__ uint4 load_shared(uint32_t smem) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4 + %5];"
                 : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(smem), "n"(OFFSET * 16));
    return r;
}
// f(0), ..., f(N - 1) with arguments known to the compiler.
template <int N, int I = 0, typename F>
__device__ __forceinline__ void unrolled(F f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        unrolled<N, I + 1>(f);
    }
}

// The share of CTA `part` of `parts` in a row.
template <int DTYPE>
struct Share {
    const uint4 *vectors;
    uint32_t head, v_lo, v_hi;
    __device__ __forceinline__ Share(const LogprobArgs &a, int64_t row, unsigned part, unsigned parts) {
        const char *row_ptr = static_cast<const char *>(a.logits) + row * a.ld * RowLayout<DTYPE>::ESIZE;
        const RowLayout<DTYPE> layout(row_ptr, static_cast<uint32_t>(a.V));
        head = layout.head;
        vectors = reinterpret_cast<const uint4 *>(row_ptr + static_cast<size_t>(head) * RowLayout<DTYPE>::ESIZE);
        const uint32_t q = layout.nvec / parts, extra = layout.nvec - q * parts;
        v_lo = q * part + min(part, extra);
        v_hi = v_lo + q + (part < extra ? 1u : 0u);
    }
    template <uint32_t PER_TRIP>
    __device__ __forceinline__ uint32_t trips() const {
        return max(1u, (v_hi - v_lo + PER_TRIP - 1) / PER_TRIP);
    }
};

// The largest of the group maxima that at least n of them reach (code of -inf or less if there is none), of
// this warp's groups.  The threads of a group -- `members` neighbours, which all hand over its maximum --
// share the comparisons out.
__device__ __forceinline__ unsigned bound_below(const float *group, int groups, unsigned members, float mine, int n) {
    const int share = groups / static_cast<int>(members);        // a multiple of 4
    const float4 *g4 = reinterpret_cast<const float4 *>(group + (threadIdx.x & (members - 1)) * share);
    int r0 = 0, r1 = 0, r2 = 0, r3 = 0;
#pragma unroll 4
    for (int o = 0; o < share / 4; ++o) {
        const float4 g = g4[o];
        r0 += g.x >= mine ? 1 : 0;
        r1 += g.y >= mine ? 1 : 0;
        r2 += g.z >= mine ? 1 : 0;
        r3 += g.w >= mine ? 1 : 0;
    }
    int reach = r0 + r1 + r2 + r3;
    for (unsigned d = 1; d < members; d <<= 1) reach += __shfl_xor_sync(0xffffffffu, reach, d);
    return __reduce_max_sync(0xffffffffu, reach >= n ? value_code(mine) : 0u);
}

// Entries of a 16-byte aligned list that are larger than `mine`.
__device__ __forceinline__ unsigned count_larger(const uint64_t *list, unsigned n, uint64_t mine) {
    unsigned r0 = 0, r1 = 0;
    const ulonglong2 *pairs = reinterpret_cast<const ulonglong2 *>(list);
#pragma unroll 8
    for (unsigned o = 0; o < n / 2; ++o) {
        const ulonglong2 q = pairs[o];
        r0 += q.x > mine ? 1u : 0u;
        r1 += q.y > mine ? 1u : 0u;
    }
    if (n & 1u) r0 += list[n - 1] > mine ? 1u : 0u;
    return r0 + r1;
}

// One CTA per row for large batches (the CTAs go on from row to row), a cluster of up to 16 CTAs per
// row for small ones: each CTA takes a share of the row's vectors and leaves its sums and
// alternatives in the shared memory of CTA 0, which merges them.  No workspace, no atomics outside a CTA,
// one launch.  (One row, no alternatives: 1 CTA 18.9 us, 8 CTAs 6.3, 16 CTAs 5.3.)
// SPLIT: whether rows are shared out.  Where they are not, everything about parts falls away at compile time: 850
// instructions per warp and row were more than a fifth of all (4096 rows of 128256 bf16: 190 us with one kernel for both, 181).
//
// Alternatives.  In the pass a thread only remembers the largest value of each of eight blocks of trips.  At
// the end of the row the top_n-th largest of 32, 64 or 128 maxima of disjoint column sets bounds the alternatives from below
// (some 24 columns reach it for top_n = 20), the blocks whose maximum reaches it are read again, spread over the
// threads, and the columns found are ranked by counting.  (Collecting candidates during the pass against a bound
// from its first trip, tightened later, cost 15 instructions a logit with the hash and 1200 cycles a trip in a
// single row.)  Rows of many equal values overflow the list: it is gathered again from the row, then without
// the bound itself, then by rounds of "largest below the last one".
template <int DTYPE, int SCHEME, bool TOP, bool SPLIT, bool LONG>
__global__ void __launch_bounds__(threads_of(SCHEME), ctas_per_sm(SCHEME))
logprob_kernel(const __grid_constant__ LogprobArgs a) {
    namespace cg = cooperative_groups;
    using Layout = RowLayout<DTYPE>;
    constexpr int VEC = Layout::VEC;
    using R = Ring<SCHEME>;
    constexpr int U = R::kGroup, kThreads = R::kThreads, kPerTrip = U * kThreads, kWarps = kThreads / 32;
    constexpr int kMostParts = SPLIT ? max_parts(TOP) : 1;
    extern __shared__ __align__(16) unsigned char sh_ring[];
    __shared__ Stats sh_warp[2][kMostParts * kWarps];            // of two rows in turn
    __shared__ RowSums sh_scratch[kWarps];
    __shared__ WarpSums sh_long[LONG ? kWarps : 1];              // of the trips before the last kChain
    __shared__ __align__(16) float sh_group[TOP ? 128 : 4];
    __shared__ unsigned sh_floor[kWarps], sh_count, sh_hits;
    __shared__ double sh_row[3];                                 // of the row being finished: largest value, ln Z, Z
    __shared__ uint16_t sh_hit[TOP ? kHits : 1];
    __shared__ float sh_block[TOP ? kBlocks : 1][kThreads];
    __shared__ __align__(16) uint64_t sh_list[TOP ? kCap : 1];
    __shared__ uint64_t sh_rounds[kWarps];
    __shared__ uint64_t sh_top[TOP ? kMaxTop : 1];               // the part's, at the end the row's alternatives in order
    __shared__ __align__(16) uint64_t sh_all[TOP && SPLIT ? kMaxTop * kMostParts : 1];  // every part's, in CTA 0

    const auto cluster = cg::this_cluster();
    const unsigned parts = SPLIT ? cluster.num_blocks() : 1u, part = SPLIT ? cluster.block_rank() : 0u;
    const uint32_t V = static_cast<uint32_t>(a.V);
    const float c = a.c;
    const unsigned tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t step = gridDim.x / parts;
    const int groups = a.top_n <= 8 ? 32 : a.top_n <= 32 ? 64 : 128;                // sets of columns whose maxima bound the alternatives
    if (parts > 1) cluster.barrier_arrive();                     // waited for before another CTA's memory is written

    if (TOP && tid == 0) sh_count = sh_hits = 0;
    const float far = 300.0f / c;
    int buf = 0;

    // The first row from r on that is not padded; what a padded row gets is written on the way.
    auto next_real = [&](int64_t r, uint32_t token) -> int64_t {
        while (r < a.B && a.tokens && token >= V) {
            if (part == 0) {
                if (tid == 0) {
                    if (a.out_logprob) a.out_logprob[r] = 0.0f;
                    if (a.out_entropy) a.out_entropy[r] = 0.0f;
                    if (a.out_rank) a.out_rank[r] = 0;
                    if (a.out_max) a.out_max[r] = 0.0f;
                    if (a.out_sumexp) a.out_sumexp[r] = 0.0f;
                }
                for (unsigned i = tid; TOP && i < static_cast<unsigned>(a.top_n); i += kThreads) {
                    if (a.out_top_ids) a.out_top_ids[r * a.top_n + i] = -1;
                    if (a.out_top_logprobs) a.out_top_logprobs[r * a.top_n + i] = -INFINITY;
                }
            }
            r += step;
            if (r < a.B) token = static_cast<uint32_t>(a.tokens[r]);
        }
        return r;
    };
    auto token_of = [&](int64_t r) -> uint32_t { return a.tokens && r < a.B ? static_cast<uint32_t>(a.tokens[r]) : 0u; };

    // The copying side: the next group's first vector of this thread, how many vectors the share has from
    // there on, and how many groups.
    const uint32_t slots = static_cast<uint32_t>(__cvta_generic_to_shared(sh_ring)) + tid * 16;
    const int64_t first_row = blockIdx.x / parts;
    int64_t src_row = first_row - step;
    const uint4 *src = nullptr;
    int src_left = 0;
    uint32_t src_groups = 0, src_slot = 0;                       // src_slot: the slot taken from last
    auto next_slot = [](uint32_t s) { return s + R::kGroupBytes == R::kBytes ? 0u : s + R::kGroupBytes; };
    auto copy_checked = [&]() {
        if (src_groups == 0) {                                   // on to the next row that is not padded
            do src_row += step;
            while (src_row != first_row && src_row < a.B && a.tokens && static_cast<uint32_t>(a.tokens[src_row]) >= V);
            src_left = 0;
            src_groups = 0xffffffffu;                            // after the last row: empty groups
            if (src_row < a.B) {
                const Share<DTYPE> share(a, src_row, part, parts);
                src = share.vectors + share.v_lo + tid;
                src_left = static_cast<int>(share.v_hi - share.v_lo - tid);
                src_groups = share.template trips<kPerTrip>();
            }
        }
        const uint32_t to = slots + src_slot;
        unrolled<U>([&](auto u) {
            constexpr int kAt = decltype(u)::value * kThreads;
            if (src_left > kAt && SBW_CHECKED(in_row(a.logits, a.ld, a.B, a.V, Layout::ESIZE, src_row, src + kAt, 16), SBW_SITE_LOGPROB_LOAD))
                copy_async<kAt>(to, src);
        });
        copy_commit();
        src += kPerTrip;
        src_left -= kPerTrip;
        --src_groups;
    };
    auto copy_first = [&]() {                                    // fills every slot but the last
#pragma unroll 1
        for (src_slot = 0; src_slot < R::kBytes - R::kGroupBytes; src_slot += R::kGroupBytes) copy_checked();
    };
    copy_first();
    uint32_t slot = 0;

    int64_t row = first_row;                                     // copied before its token was known
    uint32_t t = token_of(row);
    if (parts == 1 && a.tokens && t >= V) {                      // padded: begin again after it
        copy_wait<0>();
        src_row = first_row;
        src_groups = 0;
        copy_first();
    }
    row = next_real(row, t);
    if (row >= a.B && parts > 1) cluster.barrier_wait();

    while (row < a.B) {
        const char *row_ptr = static_cast<const char *>(a.logits) + row * a.ld * Layout::ESIZE;
        t = token_of(row);
        const uint32_t token_ahead = token_of(row + step);
        RowSeedS<SCHEME> rs;
        rs.init(a.bias.key, a.ctx + row * a.W, a.W);
        const Share<DTYPE> share(a, row, part, parts);
        const uint32_t nvec = (V - share.head) / VEC;
        // this part's columns: its vectors, the head with the first part, the tail with the last
        const uint32_t c_lo = part == 0 ? 0u : share.head + share.v_lo * VEC;
        const uint32_t c_hi = part + 1 == parts ? V : share.head + share.v_hi * VEC;

        // the ragged ends: at most one column per thread
        float xe = -INFINITY;
        uint32_t ce = V;
        if (part == 0 && tid < share.head) ce = tid;
        else if (part + 1 == parts && tid >= 32 && tid - 32 < V - share.head - nvec * VEC) ce = share.head + nvec * VEC + tid - 32;
        if (ce < V) xe = logit_at<DTYPE, SCHEME>(a, row, row_ptr, ce, rs);

        // the token's own value; its rank counts the greater ones, and the equal ones before it
        const bool ranked = a.tokens != nullptr && a.out_rank != nullptr;
        float xt = INFINITY;
        if (a.tokens) xt = logit_at<DTYPE, SCHEME>(a, row, row_ptr, t, rs);
        const bool t_nothing = ranked && !(xt > -INFINITY);
        const float bar = ranked && !t_nothing ? xt : INFINITY;

        const float below = value_below<DTYPE>(bar);             // equal ones before the token are greater than that
        const uint32_t bar2 = both_halves(bar), below2 = both_halves(below);
        const float lowest = -2.0f * a.huge;
        Stats st = {lowest * c, 0.0f, 0.0f, -INFINITY, 0u};
        float least = lowest;                                    // values below count as this
        [[maybe_unused]] uint32_t least2 = both_halves(lowest);
        uint32_t count = 0;                                      // columns that rank before the token
        [[maybe_unused]] float block_top = -INFINITY;            // largest value of the block of trips
        float2 z2 = {0.0f, 0.0f}, s2 = {0.0f, 0.0f};             // partial sums of the trip
        auto fold = [&]() {
            st.z += z2.x + z2.y;
            st.s += s2.x + s2.y;
            z2 = s2 = make_float2(0.0f, 0.0f);
        };
        // The warp's reference: its first trip's largest value, and a larger one only when some value's term is
        // more than twice that one's, so that the sums are seldom moved.  (A wider margin, 2^40, saves nothing
        // that can be measured and costs the entropy digits: S is then a difference of larger numbers.)
        float limit = lowest;
        auto raise = [&](float mx) {
            for (int d = 16; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
            fold();
            st.move(mx * c);
            least = __fsub_rd(mx, far);
            least2 = both_halves(__bfloat162float(__float2bfloat16_rd(least)));
            limit = fmaf(far, 1.0f / 300.0f, mx);                // one power of two more
        };
        auto add_pair = [&](float l0, float l1) {                // two columns in each operation
            const float2 x = __ffma2_rn(make_float2(l0, l1), make_float2(c, c), make_float2(-st.ref, -st.ref));
            const float2 e = make_float2(ex2_approx_ftz(x.x), ex2_approx_ftz(x.y));
            z2 = __fadd2_rn(z2, e);
            s2 = __ffma2_rn(e, x, s2);
        };
        uint32_t trip = 0;
        uint32_t j0 = share.v_lo + tid;                          // this trip's first vector
        const uint32_t trips = share.template trips<kPerTrip>();
        [[maybe_unused]] int block_shift = 0;                    // trips of a block: 2^block_shift
        if constexpr (TOP) {
            while (trips > static_cast<uint32_t>(kBlocks) << block_shift) ++block_shift;
        }
        auto trip_body = [&](const auto inside_tag) {
            constexpr bool INSIDE = decltype(inside_tag)::value; // this group and the one to copy now are full, of this row
            copy_wait<R::kStages - 2>();
            uint4 w[U];
            const uint32_t at = slots + slot, to = slots + src_slot;
            unrolled<U>([&](auto u) {
                constexpr int kAt = decltype(u)::value * kThreads;
                constexpr uint32_t kNone = DTYPE == SBW_DTYPE_F32 ? 0xff800000u : 0xff80ff80u;
                w[decltype(u)::value] = INSIDE || j0 + kAt < share.v_hi ? load_shared<kAt>(at) : make_uint4(kNone, kNone, kNone, kNone);
            });
            if constexpr (INSIDE) {
                unrolled<U>([&](auto u) {
                    constexpr int kAt = decltype(u)::value * kThreads;
                    if (SBW_CHECKED(in_row(a.logits, a.ld, a.B, a.V, Layout::ESIZE, row, src + kAt, 16), SBW_SITE_LOGPROB_LOAD))
                        copy_async<kAt>(to, src);
                });
                copy_commit();
                src += kPerTrip;
            } else {
                copy_checked();
            }
            src_slot = slot;
            slot = next_slot(slot);
            const uint32_t col0 = share.head + j0 * VEC;
#pragma unroll
            for (int u = 0; u < U; ++u) bias_vector<DTYPE, SCHEME>(w[u], rs, a.vocab_offset + col0 + u * (kThreads * VEC), a.bias);
            const float mx = largest_of<DTYPE, U>(w);
            st.top = fmaxf(st.top, mx);
            if (__any_sync(0xffffffffu, mx > limit)) raise(mx);
            if constexpr (TOP) {
                block_top = fmaxf(block_top, mx);
                if ((trip + 1) >> block_shift != trip >> block_shift) {
                    sh_block[trip >> block_shift][tid] = block_top;
                    block_top = -INFINITY;
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t *e = reinterpret_cast<const uint32_t *>(&w[u]);
                if constexpr (DTYPE == SBW_DTYPE_F32) {
#pragma unroll
                    for (int i = 0; i < 4; i += 2)
                        add_pair(max_nan(__uint_as_float(e[i]), least), max_nan(__uint_as_float(e[i + 1]), least));
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t q = max_nan_bf16x2(e[i], least2);
                        add_pair(__uint_as_float(q << 16), __uint_as_float(q & 0xffff0000u));
                    }
                }
            }
            if (mx >= bar) {                                     // some column may rank before the token
                if (t - col0 < static_cast<uint32_t>(((U - 1) * kThreads + 1) * VEC)) {   // the token may be among them
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const uint32_t col = col0 + u * (kThreads * VEC);
#pragma unroll
                        for (int i = 0; i < VEC; ++i) {
                            const float x = element<DTYPE>(w[u], i);
                            if (x > bar || (x == bar && col + i < t)) count += 1u;
                        }
                    }
                } else if constexpr (DTYPE == SBW_DTYPE_F32) {
                    const float over = col0 < t ? below : bar;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
#pragma unroll
                        for (int i = 0; i < VEC; ++i)
                            if (element<DTYPE>(w[u], i) > over) count += 1u;
                    }
                } else {
                    const uint32_t over = col0 < t ? below2 : bar2;
                    const __nv_bfloat162 o2 = *reinterpret_cast<const __nv_bfloat162 *>(&over);
                    const __nv_bfloat162 *q = reinterpret_cast<const __nv_bfloat162 *>(w);
                    // masks of 0xffff per half added up as words: -L in the low half after L hits there, and
                    // L - H less that borrow in the high one after H hits
                    uint32_t masks = 0;
#pragma unroll
                    for (int i = 0; i < 4 * U; ++i) masks += __hgt2_mask(q[i], o2);
                    const uint32_t low = (0u - masks) & 0xffffu;
                    count += (low + low - ((masks + low) >> 16)) & 0xffffu;
                }
            }
            fold();                                              // short chains of additions: a trip's, then the trips'
            ++trip;
            j0 += kPerTrip;
        };
        auto join_warp = [&]() {
            for (int d = 16; d > 0; d >>= 1) {
                st.z += __shfl_xor_sync(0xffffffffu, st.z, d);
                st.s += __shfl_xor_sync(0xffffffffu, st.s, d);
            }
        };
        auto end_chain = [&]() {                                 // every kChain trips, but for the row's last
            if (!LONG || trip % kChain != 0 || trip == trips) return;
            join_warp();
            if (lane == 0) {
                if (trip == kChain) sh_long[warp] = {st.z, st.s, st.ref};
                else sh_long[warp].add(st);
            }
            st.z = st.s = 0.0f;
        };
        const uint32_t full = (share.v_hi - share.v_lo) / kPerTrip;
        constexpr uint32_t kAhead = R::kStages - 1;
        if (full > kAhead) {
            const uint32_t inside = full - kAhead;               // the copies are kAhead groups ahead, in this row
            while (trip < inside) {
                trip_body(std::true_type{});
                end_chain();
            }
            src_left -= static_cast<int>(inside * kPerTrip);
            src_groups -= inside;
        }
        while (trip < trips) {
            trip_body(std::false_type{});
            end_chain();
        }
        const int64_t row_ahead = next_real(row + step, token_ahead);

        if (__any_sync(0xffffffffu, xe > limit)) raise(xe);
        if (ce < V) {
            st.top = fmaxf(st.top, xe);
            add_pair(max_nan(xe, least), 0.0f);
            z2.y = s2.y = 0.0f;
            fold();
            if (xe > bar || (xe == bar && ce < t)) count += 1u;
        }
        st.above = count;
        if (t_nothing) st.above = count_above_nothing<DTYPE, SCHEME>(a, row, c_lo, c_hi, t);

        [[maybe_unused]] const float largest = st.top;           // of the thread's columns
        if (TOP && (trip >> block_shift) < kBlocks) sh_block[trip >> block_shift][tid] = block_top;
        // ---- this warp's sums, to CTA 0 ----
        {
            for (int d = 16; d > 0; d >>= 1) st.top = fmaxf(st.top, __shfl_xor_sync(0xffffffffu, st.top, d));
            join_warp();
            if (LONG && lane == 0 && trips > kChain) {
                sh_long[warp].add(st);
                st.z = static_cast<float>(sh_long[warp].z);
                st.s = static_cast<float>(sh_long[warp].s);
            }
            st.above = __reduce_add_sync(0xffffffffu, st.above);
            if (parts > 1) cluster.barrier_wait();               // CTA 0 runs
            if (lane == 0) *cluster.map_shared_rank(&sh_warp[buf][part * kWarps + warp], 0) = st;
        }

        // ---- this part's alternatives ----
        if constexpr (TOP) {
            const unsigned need = min(static_cast<unsigned>(a.top_n), c_hi - c_lo);
            // a value that top_n columns of this part reach, from the maxima of disjoint sets of them
            const unsigned members = kThreads / groups;          // 8, 4, 2 or 1 threads
            float g = largest;
            for (unsigned d = 1; d < members; d <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, d));
            if ((tid & (members - 1)) == 0) sh_group[tid / members] = g;
            __syncthreads();
            const unsigned best = bound_below(sh_group, groups, members, g, a.top_n);
            if (lane == 0) sh_floor[warp] = best;
            __syncthreads();
            unsigned floor_code = sh_floor[0];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) floor_code = max(floor_code, sh_floor[w]);
            const float floor = __uint_as_float(order_decode(floor_code));   // -inf: perhaps fewer reach it
            const float lowest = fmaxf(floor, -FLT_MAX);
            // the columns that reach it: the vectors of a block whose maximum says there are some are read again,
            // spread over the threads
            if (ce < V && xe >= lowest) sh_list[atomicAdd(&sh_count, 1u)] = composite(xe, ce);
            unsigned in_blocks = 0;
#pragma unroll
            for (uint32_t b = 0; b < kBlocks; ++b)
                if (b << block_shift < trip && sh_block[b][tid] >= lowest) in_blocks |= 1u << b;
            if (in_blocks) {
                unsigned pos = atomicAdd(&sh_hits, static_cast<unsigned>(__popc(in_blocks)));
                for (; in_blocks; in_blocks &= in_blocks - 1, ++pos)
                    if (pos < static_cast<unsigned>(kHits)) sh_hit[pos] = static_cast<uint16_t>((__ffs(in_blocks) - 1) * kThreads + tid);
            }
            __syncthreads();
            const unsigned hits = sh_hits, per_hit = static_cast<unsigned>(U) << block_shift;
            if (hits > static_cast<unsigned>(kHits)) {
                if (tid == 0) sh_count = kCap + 1;               // too many to note: gathered from the row instead
            } else {
                for (unsigned i = tid; i < hits * per_hit; i += kThreads) {
                    const unsigned hit = sh_hit[i / per_hit];
                    const uint32_t j = share.v_lo + ((hit / kThreads) * per_hit + i % per_hit) * kThreads + hit % kThreads;
                    if (j >= share.v_hi ||
                        !SBW_CHECKED(in_row(a.logits, a.ld, a.B, a.V, Layout::ESIZE, row, share.vectors + j, 16), SBW_SITE_LOGPROB_LOAD))
                        continue;
                    uint4 v = load_vector(share.vectors + j);
                    const uint32_t col = share.head + j * VEC;
                    bias_vector<DTYPE, SCHEME>(v, rs, a.vocab_offset + col, a.bias);
                    unsigned taken = 0;
#pragma unroll
                    for (int k = 0; k < VEC; ++k) taken |= element<DTYPE>(v, k) >= lowest ? 1u << k : 0u;
                    if (taken == 0) continue;
                    unsigned pos = atomicAdd(&sh_count, static_cast<unsigned>(__popc(taken)));
#pragma unroll
                    for (int k = 0; k < VEC; ++k) {
                        if (!(taken >> k & 1u)) continue;
                        if (pos < static_cast<unsigned>(kCap)) sh_list[pos] = composite(element<DTYPE>(v, k), col + k);
                        ++pos;
                    }
                }
            }
            __syncthreads();
            unsigned n = sh_count;
            bool strict = !(floor > -INFINITY);                  // the list holds what is above the floor, not what equals it
            for (int again = 0; again < 2 && n > static_cast<unsigned>(kCap) && !(again == 1 && strict); ++again) {
                __syncthreads();                                 // everyone has read the count
                if (tid == 0) sh_count = 0;
                __syncthreads();
                strict = strict || again == 1;
                gather_again<DTYPE, SCHEME>(a, row, c_lo, c_hi, floor, strict, sh_list, &sh_count);
                __syncthreads();
                n = sh_count;
            }
            if (n > static_cast<unsigned>(kCap)) {
                select_rounds<DTYPE, SCHEME>(a, row, c_lo, c_hi, sh_top, need, sh_rounds);
            } else {
                for (unsigned i = tid; i < n; i += kThreads) {
                    const uint64_t mine = sh_list[i];
                    const unsigned rank = count_larger(sh_list, n, mine);
                    if (rank < need) {
                        if (parts > 1) *cluster.map_shared_rank(&sh_all[part * a.top_n + rank], 0) = mine;
                        else sh_top[rank] = mine;
                    }
                }
                if (n < need && warp == 0) fill_equal<DTYPE, SCHEME>(a, row, c_lo, c_hi, floor, sh_top, n, need);
            }
            if (parts > 1) {                                     // what is not there yet, and nothing for the rest
                const unsigned there = n > static_cast<unsigned>(kCap) ? 0u : min(n, need);
                if (there < need) __syncthreads();
                for (unsigned i = there + tid; i < static_cast<unsigned>(a.top_n); i += kThreads)
                    *cluster.map_shared_rank(&sh_all[part * a.top_n + i], 0) = i < need ? sh_top[i] : 0;
            }
        }
        if (parts > 1) cluster.sync();                           // everything has arrived in CTA 0
        else if (!TOP) __syncthreads();

        // ---- the row ----
        const Stats *sums = sh_warp[buf];
        const unsigned n_sums = parts * kWarps;
        float m = -INFINITY;                                     // the row's largest value
        if (part == 0) {
            for (unsigned i = lane; i < n_sums; i += 32) m = fmaxf(m, sums[i].top);
            for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
        }
        const bool nothing = m == -INFINITY, ordinary = fabsf(m) < a.huge;
        RowSums plain = {};
        if (part == 0 && !nothing && !ordinary) plain = sum_plainly<DTYPE, SCHEME>(a, row, 0u, V, m, sh_scratch);
        if (part == 0 && warp == kWarps - 1) {
            double z = 0.0, s = 0.0;
            uint32_t above = 0;
            const float ref = ordinary ? m * c : 0.0f;
            for (unsigned i = lane; i < n_sums; i += 32) {
                Stats p = sums[i];
                above += p.above;
                p.move(ref);
                z += static_cast<double>(p.z);
                s += static_cast<double>(p.s);
            }
            for (int d = 16; d > 0; d >>= 1) {
                z += __shfl_xor_sync(0xffffffffu, z, d);
                s += __shfl_xor_sync(0xffffffffu, s, d);
            }
            above = __reduce_add_sync(0xffffffffu, above);
            if (nothing) {
                z = z == z ? 0.0 : z;                            // NaN and -inf alone: NaN
            } else if (ordinary) {
                // relative to m itself from here on: the terms are 2^((l - m) c) 2^(m c - ref)
                const double d = static_cast<double>(m) * static_cast<double>(c) - static_cast<double>(ref);
                s -= d * z;
                const double y = -0.6931471805599453 * d;        // tiny unless m c is huge
                const double f = fabs(y) < 1e-4 ? 1.0 + y * (1.0 + 0.5 * y) : exp(y);
                z *= f;
                s *= f;
            } else {
                z = plain.z;
                s = plain.s;
            }
            z -= a.c_off * s;                                    // c was rounded: to first order, 2^(x off) = 1 + x off ln 2
            const double ln_z = log(z);
            if (lane == 0) {
                const bool empty = z == 0.0;                     // every logit is -inf
                if (SBW_CHECKED(row >= 0 && row < a.B && above < V, SBW_SITE_LOGPROB_OUTPUT)) {
                    if (a.out_logprob)
                        a.out_logprob[row] = empty ? -INFINITY : static_cast<float>((static_cast<double>(xt) - m) * a.inv_tau - ln_z);
                    if (a.out_entropy) a.out_entropy[row] = empty ? 0.0f : static_cast<float>(ln_z - 0.6931471805599453 * s / z);
                    if (a.out_rank) a.out_rank[row] = 1 + static_cast<int32_t>(above);
                    if (a.out_max) a.out_max[row] = z != z ? NAN : m;                // NaN: a NaN or +inf among the logits
                    if (a.out_sumexp) a.out_sumexp[row] = static_cast<float>(z);
                }
                if (TOP) {
                    sh_row[0] = m;
                    sh_row[1] = ln_z;
                    sh_row[2] = z;
                }
            }
        }
        if constexpr (TOP) {
            if (part == 0) {
                const unsigned n = a.top_n;
                if (parts > 1) {                                 // the parts' lists into one
                    for (unsigned i = tid; i < n * parts; i += kThreads) {
                        const uint64_t mine = sh_all[i];
                        const unsigned rank = mine ? count_larger(sh_all, n * parts, mine) : n;
                        if (rank < n) sh_top[rank] = mine;
                    }
                }
                __syncthreads();
                if (tid == 0) sh_count = sh_hits = 0;            // for the next row, whose first barrier comes before any use
                for (unsigned i = tid; i < n; i += kThreads) {
                    const uint64_t mine = i < V ? sh_top[i] : 0;
                    const double lp = (static_cast<double>(composite_value(mine)) - sh_row[0]) * a.inv_tau - sh_row[1];
                    if (a.out_top_ids) a.out_top_ids[row * n + i] = i < V ? static_cast<int32_t>(0xFFFFFFFFu - static_cast<uint32_t>(mine)) : -1;
                    if (a.out_top_logprobs)
                        a.out_top_logprobs[row * n + i] = i >= V || sh_row[2] == 0.0 ? -INFINITY : static_cast<float>(lp);
                }
            }
        }
        buf ^= 1;
        row = row_ahead;
    }
    copy_wait<0>();
}

// Gradient: no reduction, so a row is cut into blocks of kGradVectors vectors per thread and every block works
// alone.  Without the hash a thread has all its loads in flight at once; with it the vectors are taken one by one
// (the loop's code, eight hash chains long, then fits the instruction cache) and the next one is loaded
// while one is hashed.
constexpr int kGradThreads = 128;
constexpr int kGradVectors = 8;

struct GradArgs {
    const void *logits;
    void *grad;
    int64_t B, V, ld, grad_ld;
    const int32_t *ctx;
    int W;
    uint32_t vocab_offset;
    BiasParams bias;
    double tau;
    float c;
    const int32_t *tokens;
    const float *max, *sumexp, *entropy, *grad_logprob, *grad_entropy;
    uint32_t blocks_per_row;
};

// What a row's elements need:  dl = -e (base + slope x), e = 2^x, x = (l - m) c, and the token's own
// share on top.
struct GradRow {
    float m, c, base, slope, own;
    uint32_t t;
    __device__ __forceinline__ float at(float l) const {
        const float x = max_nan((l - m) * c, kFar);
        return -ex2_approx_ftz(x) * fmaf(slope, x, base);
    }
};

template <int DTYPE>
__device__ __forceinline__ void store_one(char *row, uint32_t col, float g) {
    if constexpr (DTYPE == SBW_DTYPE_F32) reinterpret_cast<float *>(row)[col] = g;
    else reinterpret_cast<__nv_bfloat16 *>(row)[col] = __float2bfloat16_rn(g);
}

template <int DTYPE, int SCHEME>
__global__ void __launch_bounds__(kGradThreads)
logprob_backward_kernel(const GradArgs a) {
    using Layout = RowLayout<DTYPE>;
    constexpr int VEC = Layout::VEC;
    const int64_t row = blockIdx.x / a.blocks_per_row;
    const uint32_t block = blockIdx.x % a.blocks_per_row;
    const uint32_t V = static_cast<uint32_t>(a.V);
    const char *row_ptr = static_cast<const char *>(a.logits) + row * a.ld * Layout::ESIZE;
    char *out_ptr = static_cast<char *>(a.grad) + row * a.grad_ld * Layout::ESIZE;
    const Layout layout(row_ptr, V);
    const uint4 *vectors = reinterpret_cast<const uint4 *>(row_ptr + static_cast<size_t>(layout.head) * Layout::ESIZE);
    char *out_vectors = out_ptr + static_cast<size_t>(layout.head) * Layout::ESIZE;
    const bool same_phase = (reinterpret_cast<uintptr_t>(out_vectors) & 15u) == 0;

    const uint32_t t = a.tokens ? static_cast<uint32_t>(a.tokens[row]) : 0xFFFFFFFFu;
    const bool padded = a.tokens && t >= V;
    const uint32_t first = block * (kGradThreads * kGradVectors) + threadIdx.x;
    const uint32_t end = min(layout.nvec, (block + 1) * (kGradThreads * kGradVectors));
    constexpr int kHeld = SCHEME == kSchemeNone ? kGradVectors : 1;
    uint4 w[kHeld];
    if (!padded) {
#pragma unroll
        for (int u = 0; u < kHeld; ++u)
            if (first + u * kGradThreads < end &&
                SBW_CHECKED(in_row(a.logits, a.ld, a.B, a.V, Layout::ESIZE, row, vectors + first + u * kGradThreads, 16), SBW_SITE_GRAD_LOAD))
                w[u] = load_vector(vectors + first + u * kGradThreads);
    }
    // the row's factors, in fp64 by one thread while the logits arrive
    __shared__ GradRow sh_row;
    __shared__ bool sh_zero;
    if (threadIdx.x == 0) {
        GradRow r = {0.0f, a.c, 0.0f, 0.0f, 0.0f, 0xFFFFFFFFu};
        bool zero = padded;
        if (!padded) {
            const double z = a.sumexp[row];
            if (z == 0.0) {                              // every logit is -inf: nothing to move
                zero = true;
            } else {
                const double g = a.grad_logprob ? a.grad_logprob[row] : 0.0;
                const double h = a.grad_entropy ? a.grad_entropy[row] : 0.0;
                const double scale = 1.0 / (a.tau * z);
                r.m = a.max[row];
                // ln p + H = x ln 2 - ln Z + H
                r.base = static_cast<float>(scale * (g + (a.grad_entropy ? h * (a.entropy[row] - log(z)) : 0.0)));
                r.slope = static_cast<float>(scale * h * 0.6931471805599453);
                r.own = static_cast<float>(g / a.tau);
                r.t = t;
            }
        }
        sh_row = r;
        sh_zero = zero;
    }
    RowSeedS<SCHEME> rs;
    if (!padded) rs.init(a.bias.key, a.ctx + row * a.W, a.W);
    __syncthreads();
    const GradRow r = sh_row;
    const bool zero = sh_zero;
    auto emit = [&](uint4 v, uint32_t j) {               // the gradient of vector j
        if (!SBW_CHECKED(in_row(a.grad, a.grad_ld, a.B, a.V, Layout::ESIZE, row, out_vectors + static_cast<size_t>(j) * 16, 16), SBW_SITE_GRAD_STORE))
            return;
        const uint32_t col = layout.head + j * VEC;
        float g[VEC];
        if (zero) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) g[i] = 0.0f;
        } else {
            bias_vector<DTYPE, SCHEME>(v, rs, a.vocab_offset + col, a.bias);
#pragma unroll
            for (int i = 0; i < VEC; ++i) g[i] = r.at(element<DTYPE>(v, i));
            if (r.t - col < static_cast<uint32_t>(VEC)) {
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (col + i == r.t) g[i] += r.own;
            }
        }
        if (same_phase) {
            uint4 o;
            uint32_t *e = reinterpret_cast<uint32_t *>(&o);
            if constexpr (DTYPE == SBW_DTYPE_F32) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) e[i] = __float_as_uint(g[i]);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; i += 2) {
                    const __nv_bfloat162 p = __floats2bfloat162_rn(g[i], g[i + 1]);
                    e[i / 2] = *reinterpret_cast<const uint32_t *>(&p);
                }
            }
            __stcs(reinterpret_cast<uint4 *>(out_vectors) + j, o);   // not read again here: leave L2 to the loads
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) store_one<DTYPE>(out_ptr, col + i, g[i]);
        }
    };
    if constexpr (SCHEME == kSchemeNone) {
#pragma unroll
        for (int u = 0; u < kGradVectors; ++u)
            if (first + u * kGradThreads < end) emit(w[u], first + u * kGradThreads);
    } else {
#pragma unroll 1
        for (uint32_t j = first; j < end; j += kGradThreads) {
            const uint4 v = w[0];
            if (!padded && j + kGradThreads < end &&
                SBW_CHECKED(in_row(a.logits, a.ld, a.B, a.V, Layout::ESIZE, row, vectors + j + kGradThreads, 16), SBW_SITE_GRAD_LOAD))
                w[0] = load_vector(vectors + j + kGradThreads);
            emit(v, j);
        }
    }
    if (block == 0) {                                    // ragged ends
        const uint32_t first_tail = layout.head + layout.nvec * VEC;
        uint32_t col = V;
        if (threadIdx.x < layout.head) col = threadIdx.x;
        else if (threadIdx.x >= 32 && threadIdx.x - 32 < V - first_tail) col = first_tail + threadIdx.x - 32;
        if (col < V) {
            const size_t at = static_cast<size_t>(col) * Layout::ESIZE;
            float g = 0.0f;
            if (!zero && SBW_CHECKED(in_row(a.logits, a.ld, a.B, a.V, Layout::ESIZE, row, row_ptr + at, Layout::ESIZE), SBW_SITE_GRAD_LOAD))
                g = r.at(biased_at<DTYPE, SCHEME>(row_ptr, col, rs, a.vocab_offset + col, a.bias));
            if (!zero && col == r.t) g += r.own;
            if (SBW_CHECKED(in_row(a.grad, a.grad_ld, a.B, a.V, Layout::ESIZE, row, out_ptr + at, Layout::ESIZE), SBW_SITE_GRAD_STORE))
                store_one<DTYPE>(out_ptr, col, g);
        }
    }
}

// ---- host side ----
struct Common {
    const void *logits;
    int dtype;
    int64_t B, V, ld, vocab_offset;
    const int32_t *ctx_tokens;
    int ctx_width;
    uint64_t key;
    double gamma;
    float delta;
    int scheme;
    float temperature;
};

// Argument checks both calls share; `marked` says whether the watermark changes any logit.
int check_common(const Common &q, bool *marked) {
    if (!valid_common(q.dtype, q.ctx_width, q.gamma, q.scheme)) return SBW_ERR_INVALID_ARG;
    if (q.B < 0 || q.V <= 0 || q.ld < q.V || q.vocab_offset < 0) return SBW_ERR_INVALID_ARG;
    if (!(q.temperature > 0.0f) || q.temperature - q.temperature != 0.0f) return SBW_ERR_INVALID_ARG;
    if (!(q.delta == q.delta) || q.delta - q.delta != 0.0f) return SBW_ERR_INVALID_ARG;
    const double c = 1.4426950408889634 / static_cast<double>(q.temperature);
    if (!(c > 1.4e-6 && c < 1.5e6)) return SBW_ERR_INVALID_ARG;    // temperature outside 1e-6 .. 1e6
    if (q.V > 0x7fffffffLL || q.vocab_offset + q.V > (int64_t(1) << 32)) return SBW_ERR_UNSUPPORTED;
    const float in_precision = q.dtype == SBW_DTYPE_BF16 ? __bfloat162float(__float2bfloat16_rn(q.delta)) : q.delta;
    *marked = in_precision != 0.0f;
    if (q.B == 0) return SBW_OK;
    if (!q.logits || (*marked && !q.ctx_tokens)) return SBW_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(q.logits) % (q.dtype == SBW_DTYPE_F32 ? 4 : 2) != 0) return SBW_ERR_INVALID_ARG;
    return SBW_OK;
}

BiasParams bias_params(const Common &q) {
    BiasParams p;
    p.key = q.key;
    p.thr_m1 = threshold_minus_one(q.gamma);
    p.delta = q.delta;
    p.delta_bf16 = 0;
    if (q.dtype == SBW_DTYPE_BF16) {
        const __nv_bfloat16 d = __float2bfloat16_rn(q.delta);
        p.delta_bf16 = static_cast<uint32_t>(__bfloat16_as_ushort(d));
        p.delta = __bfloat162float(d);
    }
    p.weyl = make_weyl();
    return p;
}

// CTAs per row, so that few rows still fill the GPU: as many as are resident at once, or with the hash the next
// whole number above that (256 x 151936 fp32 self-salt: 2 CTAs 227 us, 3 218, where 2.3 would be resident; no rule was found
// in 4 to 8 CTAs: 220, 216, 207, 223, 219); but no more than find a trip each, and up to 8 -- larger clusters leave
// SMs of a GPC unused -- but for a handful of rows (one row without alternatives: 8 CTAs 6.3 us, 16 CTAs 5.3).
int parts_per_row(int64_t B, int64_t nvec, int64_t per_trip, int sm_count, int scheme, int most_parts) {
    const int64_t slots = static_cast<int64_t>(sm_count) * ctas_per_sm(scheme);
    int64_t parts = scheme < 0 ? slots / B : (slots + B - 1) / B;
    const int64_t trips = (nvec + per_trip - 1) / per_trip;
    const int64_t most = B <= 8 ? most_parts : 8;
    if (parts > most) parts = most;
    if (parts > trips) parts = trips;
    return static_cast<int>(parts < 1 ? 1 : parts);
}

template <int DTYPE, int SCHEME, bool TOP, bool SPLIT, bool LONG>
int launch_logprobs(const LogprobArgs &a, int parts, const DeviceInfo &di, cudaStream_t s) {
    using R = Ring<SCHEME>;
    const auto kernel = logprob_kernel<DTYPE, SCHEME, TOP, SPLIT, LONG>;
    // clusters above 8 CTAs and that much shared memory have to be asked for, once per device
    static std::atomic<uint64_t> prepared{0};
    if (!(prepared.load(std::memory_order_acquire) >> di.device & 1)) {
        if (SPLIT) SBW_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        SBW_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, R::kBytes));
        prepared.fetch_or(uint64_t(1) << di.device, std::memory_order_release);
    }
    const int64_t resident = static_cast<int64_t>(di.sm_count) * ctas_per_sm(SCHEME);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(SPLIT ? a.B * parts : (a.B < resident ? a.B : resident)));
    cfg.blockDim = dim3(R::kThreads);
    cfg.dynamicSmemBytes = R::kBytes;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(parts);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = SPLIT ? 1 : 0;
    SBW_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a));
    return SBW_OK;
}

template <int DTYPE, int SCHEME, bool TOP>
int launch_logprobs(const LogprobArgs &a, cudaStream_t s) {
    DeviceInfo di;
    if (int rc = current_device_info(&di)) return rc;
    if (di.device >= 64) return SBW_ERR_UNSUPPORTED;
    constexpr int64_t per_trip = Ring<SCHEME>::kGroup * Ring<SCHEME>::kThreads;
    const int64_t nvec = a.V / RowLayout<DTYPE>::VEC;            // of a row, at most
    const int parts = parts_per_row(a.B, nvec, per_trip, di.sm_count, SCHEME, max_parts(TOP));
    const bool is_long = (nvec + parts - 1) / parts > kChain * per_trip;
    if (parts > 1)
        return is_long ? launch_logprobs<DTYPE, SCHEME, TOP, true, true>(a, parts, di, s)
                       : launch_logprobs<DTYPE, SCHEME, TOP, true, false>(a, parts, di, s);
    return is_long ? launch_logprobs<DTYPE, SCHEME, TOP, false, true>(a, parts, di, s)
                   : launch_logprobs<DTYPE, SCHEME, TOP, false, false>(a, parts, di, s);
}

template <int DTYPE, int SCHEME>
int launch_logprobs(const LogprobArgs &a, cudaStream_t s) {
    return a.top_n > 0 ? launch_logprobs<DTYPE, SCHEME, true>(a, s) : launch_logprobs<DTYPE, SCHEME, false>(a, s);
}

template <int DTYPE>
int launch_logprobs(const LogprobArgs &a, bool marked, int scheme, cudaStream_t s) {
    if (!marked) return launch_logprobs<DTYPE, kSchemeNone>(a, s);
    return scheme == SBW_SCHEME_CONTEXT ? launch_logprobs<DTYPE, SBW_SCHEME_CONTEXT>(a, s)
                                        : launch_logprobs<DTYPE, SBW_SCHEME_SELFSALT>(a, s);
}

template <int DTYPE, int SCHEME>
int launch_backward(const GradArgs &a, int64_t blocks, cudaStream_t s) {
    logprob_backward_kernel<DTYPE, SCHEME><<<static_cast<unsigned>(blocks), kGradThreads, 0, s>>>(a);
    SBW_CUDA_TRY(cudaGetLastError());
    return SBW_OK;
}

template <int DTYPE>
int launch_backward(const GradArgs &a, int64_t blocks, bool marked, int scheme, cudaStream_t s) {
    if (!marked) return launch_backward<DTYPE, kSchemeNone>(a, blocks, s);
    return scheme == SBW_SCHEME_CONTEXT ? launch_backward<DTYPE, SBW_SCHEME_CONTEXT>(a, blocks, s)
                                        : launch_backward<DTYPE, SBW_SCHEME_SELFSALT>(a, blocks, s);
}

// Whether a [B, V] block with row stride ld_a at `a` and one with ld_b at `b` share an element (in
// units of elements).  The same block in both places is the caller's in-place call, judged before.
bool blocks_overlap(uintptr_t a, int64_t ld_a, uintptr_t b, int64_t ld_b, int64_t B, int64_t V, int esize) {
    const uintptr_t end_a = a + static_cast<uintptr_t>((B - 1) * ld_a + V) * esize;
    const uintptr_t end_b = b + static_cast<uintptr_t>((B - 1) * ld_b + V) * esize;
    if (end_a <= b || end_b <= a) return false;
    if (ld_a != ld_b) return true;                       // interleaved with different strides: not told apart, refused
    const uintptr_t apart = b > a ? b - a : a - b;
    const uintptr_t stride = static_cast<uintptr_t>(ld_a) * esize, width = static_cast<uintptr_t>(V) * esize;
    const uintptr_t r = apart % stride;                  // rows of one lie in the gaps of the other?
    return r < width || stride - r < width;
}

}  // namespace
}  // namespace sbw

extern "C" int sbw_token_logprobs(const void *logits, int dtype, int64_t B, int64_t V, int64_t ld, int64_t vocab_offset,
                                  const int32_t *ctx_tokens, int ctx_width, uint64_t key, double gamma, float delta,
                                  int scheme, float temperature, const int32_t *tokens, int64_t top_n,
                                  float *out_logprob, float *out_entropy, int32_t *out_rank, float *out_max,
                                  float *out_sumexp, int32_t *out_top_ids, float *out_top_logprobs, void *stream) {
    using namespace sbw;
    const Common q = {logits, dtype, B, V, ld, vocab_offset, ctx_tokens, ctx_width, key, gamma, delta, scheme, temperature};
    bool marked = false;
    if (top_n < 0) return SBW_ERR_INVALID_ARG;
    if (int rc = check_common(q, &marked)) return rc;
    if (top_n > SBW_MAX_TOP_LOGPROBS) return SBW_ERR_TOO_LARGE;
    if (B == 0) return SBW_OK;
    if (!tokens && (out_logprob || out_rank)) return SBW_ERR_INVALID_ARG;
    if (top_n == 0 ? (out_top_ids || out_top_logprobs) : (!out_top_ids && !out_top_logprobs)) return SBW_ERR_INVALID_ARG;
    if (!out_logprob && !out_entropy && !out_rank && !out_max && !out_sumexp && top_n == 0) return SBW_ERR_INVALID_ARG;
    LogprobArgs a;
    a.logits = logits;
    a.B = B; a.V = V; a.ld = ld;
    a.ctx = ctx_tokens;
    a.W = ctx_width;
    a.vocab_offset = static_cast<uint32_t>(vocab_offset);
    a.bias = bias_params(q);
    a.inv_tau = 1.0 / static_cast<double>(temperature);
    const double c = 1.4426950408889634 / static_cast<double>(temperature);
    a.c = static_cast<float>(c);
    a.c_off = 0.6931471805599453 * (static_cast<double>(a.c) / c - 1.0);
    a.huge = __bfloat162float(__float2bfloat16_rz(static_cast<float>(kOrdinary / c)));
    a.tokens = tokens;
    a.top_n = static_cast<int>(top_n);
    a.out_logprob = out_logprob;
    a.out_entropy = out_entropy;
    a.out_rank = out_rank;
    a.out_max = out_max;
    a.out_sumexp = out_sumexp;
    a.out_top_ids = out_top_ids;
    a.out_top_logprobs = out_top_logprobs;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return dtype == SBW_DTYPE_F32 ? launch_logprobs<SBW_DTYPE_F32>(a, marked, scheme, s)
                                  : launch_logprobs<SBW_DTYPE_BF16>(a, marked, scheme, s);
}

extern "C" int sbw_token_logprobs_backward(const void *logits, int dtype, int64_t B, int64_t V, int64_t ld,
                                           int64_t vocab_offset, const int32_t *ctx_tokens, int ctx_width, uint64_t key,
                                           double gamma, float delta, int scheme, float temperature,
                                           const int32_t *tokens, const float *max, const float *sumexp,
                                           const float *entropy, const float *grad_logprob, const float *grad_entropy,
                                           void *grad_logits, int64_t grad_ld, void *stream) {
    using namespace sbw;
    const Common q = {logits, dtype, B, V, ld, vocab_offset, ctx_tokens, ctx_width, key, gamma, delta, scheme, temperature};
    bool marked = false;
    if (grad_ld < V) return SBW_ERR_INVALID_ARG;
    if (int rc = check_common(q, &marked)) return rc;
    if (B == 0) return SBW_OK;
    if (!max || !sumexp || !grad_logits) return SBW_ERR_INVALID_ARG;
    if ((!grad_logprob && !grad_entropy) || (grad_logprob && !tokens) || (grad_entropy && !entropy)) return SBW_ERR_INVALID_ARG;
    const int esize = dtype == SBW_DTYPE_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(grad_logits) % esize != 0) return SBW_ERR_INVALID_ARG;
    const bool in_place = grad_logits == logits && grad_ld == ld;
    if (!in_place && blocks_overlap(reinterpret_cast<uintptr_t>(logits), ld, reinterpret_cast<uintptr_t>(grad_logits), grad_ld, B, V, esize))
        return SBW_ERR_INVALID_ARG;
    const int64_t per_block = static_cast<int64_t>(kGradThreads) * kGradVectors * (16 / esize);
    const int64_t per_row = (V + per_block - 1) / per_block;
    if (B > 0x7fffffffLL / per_row) return SBW_ERR_UNSUPPORTED;
    GradArgs a;
    a.logits = logits;
    a.grad = grad_logits;
    a.B = B; a.V = V; a.ld = ld; a.grad_ld = grad_ld;
    a.ctx = ctx_tokens;
    a.W = ctx_width;
    a.vocab_offset = static_cast<uint32_t>(vocab_offset);
    a.bias = bias_params(q);
    a.tau = static_cast<double>(temperature);
    a.c = static_cast<float>(1.4426950408889634 / static_cast<double>(temperature));
    a.tokens = tokens;
    a.max = max;
    a.sumexp = sumexp;
    a.entropy = entropy;
    a.grad_logprob = grad_logprob;
    a.grad_entropy = grad_entropy;
    a.blocks_per_row = static_cast<uint32_t>(per_row);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return dtype == SBW_DTYPE_F32 ? launch_backward<SBW_DTYPE_F32>(a, B * per_row, marked, scheme, s)
                                  : launch_backward<SBW_DTYPE_BF16>(a, B * per_row, marked, scheme, s);
}
