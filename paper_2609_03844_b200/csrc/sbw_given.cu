// sbw_sample_given: one token per row of (watermarked) logits from a given random number, with a
// temperature, top-k, top-p and min-p of its own for every row.
//
// The candidates of a row are ordered by value, descending, equal ones by column; the filters keep a
// prefix of that order, and the token is the first candidate at which the running weight passes the
// given share of what is kept.  Weights are the integers of sbw_bias_sample_filtered (2^40 for the
// maximum), so that every sum is exact and no result depends on an order of addition.  So there is one
// question, asked up to three times per row: at which candidate does the running number (top-k) or the
// running weight (top-p, then the draw) reach a target?
//
// A row belongs to one CTA, or to a cluster of up to 8 where that many CTAs for every row are under way at once, and, watermarked
// in fp32, where a CTA has no room for its part (from 17408 logits on: 128256 are 8 CTAs at any batch).  Two ways of doing it:
//   by value    (bf16) few values are distinct: one pass counts them, before the maximum is known; weights and all three
//               questions are then a matter of the counters, and a second pass, from L2, finds the column.
//   by weight   (fp32, and the bf16 rows that the counters do not hold, such as those with a maximum around 0)
//     maximum    one pass
//     histogram  1024 bins by the weight's exponent and six bits of its mantissa, down to 2^-16 of the maximum: the
//                number of candidates and the sum of the other 17 bits (32-bit counters, native adds).  Weights below
//                that are summed in registers.
//     lists      the first CTA scans the bins, asks all for the candidates of the first bins up to the one that is looked
//                for (of that bin alone if those are too many for the list), sorts them and walks the running sums.  The
//                first list usually answers all questions.
//     A bin too full for the list is split by the candidates' bits, 1024 ways at a time; candidates of equal value,
//     however many, are counted by column.  Rows are read again by every pass, watermarked bf16 ones hashed again;
//     watermarked fp32 ones stay in the cluster's shared memory.
// Measured on 1024 x 128256, repeated calls: bf16 166 us, where the bytes take 40; the counting pass's 21 instructions for 32
// logits, half of them on the ALU pipe, and its adds to shared memory bound it.  fp32 with top-p 0.9 422 us, where the bytes take 80
// and the three readings, of rows that L2 does not hold, 240; the passes' instructions (45 for 32 logits) and a row's serial
// phases are the rest.  A row that draws a candidate below 2^-16 of its maximum is slow, since a split of the tail handles each of
// its candidates by itself: 256 x 128256 with no filter 97 us with every random number 0.5, 967 where one is 0.99999.  bf16 rows
// with a maximum of 0 are counted first and then done by weight: 1024 x 128256 403 us with top-p 0.9.
#include <atomic>
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "sbw_codes.cuh"
#include "sbw_common.cuh"
#include "sbw_hash.cuh"
#include "sbw_rowbias.cuh"

namespace sbw {
namespace {

namespace cg = cooperative_groups;

constexpr int kGivenThreads = 512;
constexpr int kGivenWarps = kGivenThreads / 32;
// A weight as fp32 bits: 2^40 has exponent 167.  Bins are the bits from the 17th up, counted so that the
// maximum's is the last one; below the first lies the tail.  The polynomial of the weights is monotone at
// that resolution (all fp32 arguments were tried; at one bit more it is not), so bins keep the order.
constexpr int kLowBits = 17;
constexpr int kBins = 1024;
constexpr uint32_t kFirstBits = (167u << (23 - kLowBits)) - (kBins - 1);
constexpr int kTail = -1;                  // number of the bin of everything below
constexpr int kFine = 1024;                // bins of a split
constexpr int kListCap = 2048;
constexpr int kCountingSort = 128;         // a list up to this length is sorted by counting
constexpr int kPrefixCap = 1024;           // a list from the first candidate on is made up to this length
constexpr int kMaxParts = 8;
constexpr int64_t kMaxGivenV = 320 * 1024;
// Of a resident row in a CTA's shared memory, before more CTAs share it.  The size hardly matters: 64 x 128256 fp32
// watermarked takes 123 us with 34 or 68 KB and 121 with 136, 256 x 151936 467 with each.
constexpr int64_t kSliceBytes = 68 * 1024;
// A sum of 17 bits holds 32768 candidates: of a resident part every other warp has its own, of a streamed row every warp.
static_assert(kMaxGivenV / kMaxParts / 2 + 8 * kGivenThreads <= 32768 && kSliceBytes / 4 / 2 + 8 * kGivenThreads <= 32768, "");
static_assert(kMaxGivenV / kGivenWarps + 8 * 32 + 16 <= 32768, "");
constexpr uint32_t kLimb = 12;                       // of a split's two sums

struct GivenArgs {
    const void *logits;
    int64_t B, V, ld;
    uint32_t vocab_offset;
    const int32_t *ctx;
    int W;
    BiasParams bias;
    const float *uniforms, *temperature;
    const int32_t *top_k;      // this and the next two: nullptr = off for every row
    const float *top_p, *min_p;
    int32_t *out_tokens;
    float *out_prob;           // nullable, and the next
    int32_t *out_kept;
    uint32_t parts;            // CTAs per row
    uint32_t part_vectors;     // 16-byte vectors of a row per CTA
};

enum { kDone = 0, kGather, kSplit, kCountTies, kPickTie };
struct Command {
    int op;
    int bin_lo, bin_hi;        // kGather, kSplit: candidates of these bins ...
    uint32_t dist_lo, dist_hi; // ... whose distance below the maximum (in codes) lies here; ties: dist_lo alone
    uint32_t shift;            // kSplit: distance - dist_lo, by this many bits to the right, is the bin
    uint32_t part, which;      // kPickTie
};

struct Sums {
    unsigned long long weight;
    uint32_t n;
};
struct ScanSlots {
    unsigned long long weight[kGivenWarps];
    uint32_t n[kGivenWarps];
};
// What a row asks for.
struct Settings {
    float c, lowest;           // as in RowWeights
    int64_t top_k;             // 0: off
    uint64_t p32;              // 0: off
    uint32_t u32;
    Settings() = default;
    __device__ __forceinline__ Settings(const GivenArgs &a, int64_t row) {
        if (!SBW_CHECKED(row >= 0 && row < a.B, SBW_SITE_GIVEN_LOAD)) {
            *this = Settings{};
            return;
        }
        const float tau = a.temperature[row];
        const bool greedy = !(tau >= 1e-6f);
        c = greedy ? 1.0f : static_cast<float>(1.4426950408889634 / static_cast<double>(tau));
        lowest = -40.0f;                                 // below that a weight is 0
        if (!greedy && a.min_p && a.min_p[row] > 0.0f)
            lowest = fminf(fmaxf(static_cast<float>(log2(static_cast<double>(a.min_p[row]))), -40.0f), 0.0f);
        top_k = greedy ? 1 : a.top_k ? a.top_k[row] : 0;
        p32 = 0;
        if (!greedy && a.top_p && a.top_p[row] < 1.0f) {
            const double p = floor(static_cast<double>(a.top_p[row]) * 4294967296.0);
            p32 = p >= 1.0 ? static_cast<uint64_t>(p) : 1ull;
        }
        const double u = static_cast<double>(a.uniforms[row]) * 4294967296.0;
        u32 = u >= 4294967295.0 ? 0xffffffffu : u >= 1.0 ? static_cast<uint32_t>(u) : 0u;
    }
};

template <int COPIES>
struct GivenShared {
    struct {
        uint32_t n[kBins], low[COPIES][kBins];
    } hist;                                           // a CTA's own candidates
    struct {
        unsigned long long weight[kBins];
        uint32_t n[kBins];
    } bins;                                           // first CTA: the row's
    union {
        unsigned long long list[kListCap];
        struct {
            uint32_t n[kFine], lo[kFine], hi[kFine];
        } fine;
    };
    ScanSlots scan;
    unsigned long long found_before, found_weight;    // running weight before, own weight
    unsigned long long tail_weight[kMaxParts];
    uint32_t tail_n[kMaxParts];
    float part_max[kMaxParts];
    uint32_t ties[kMaxParts];
    uint32_t tie_col;
    uint32_t list_n, list_at;
    int found_at;
    uint32_t found_n_before, found_n;
    uint32_t found_dist, found_col;
    float warp_max[kGivenWarps];
    Settings set;
    Command cmd;
};

// What a row's weights depend on.
struct RowWeights {
    float m, c, lowest;        // maximum; log2(e) / temperature; least log2 of a kept weight over the maximum's
    uint32_t code_m;
    __device__ __forceinline__ float log2_of(float x) const { return __fmul_rn(__fsub_rn(x, m), c); }
};

// Two fp32 operations per instruction.
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair_of(float a, float b) {
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(a), "f"(b));
    return p;
}
__device__ __forceinline__ void of_pair(Pair p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ Pair pair_add(Pair a, Pair b) {
    Pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ Pair pair_mul(Pair a, Pair b) {
    Pair d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ Pair pair_fma(Pair a, Pair b, Pair c) {
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

// 2^(40 + y) as fp32 for two y in [-41, 0]; anything for others.  The steps and coefficients are those of the
// weights of sbw_bias_sample_filtered, the latter times 2^40: a power of two changes no rounding.  The weight is what
// truncation leaves of it.
constexpr float kRound = 12582912.0f;                // 1.5 2^23: the last bits of y + kRound are rint(y)
// N pairs side by side: a step's constant, which takes two registers, is made once for all of them.
template <int N>
__device__ __forceinline__ void power(const Pair (&y)[N], uint32_t (&v)[2 * N]) {
    constexpr float kSteps[7] = {0x1.430912p+27f, 0x1.5d87fep+30f, 0x1.3b2ab6p+33f, 0x1.c6b08ep+35f, 0x1.ebfbep+37f, 0x1.62e43p+39f, 0x1p+40f};
    Pair t[N], f[N], p[N];
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = pair_add(y[i], pair_of(kRound, kRound));
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = pair_add(t[i], pair_of(-kRound, -kRound));
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = pair_fma(f[i], pair_of(-1.0f, -1.0f), y[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = pair_of(0x1.ffcbfcp+23f, 0x1.ffcbfcp+23f);
#pragma unroll
    for (int k = 0; k < 7; ++k) {
        const Pair c = pair_of(kSteps[k], kSteps[k]);
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = pair_fma(p[i], f[i], c);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float p0, p1, t0, t1;
        of_pair(p[i], p0, p1);
        of_pair(t[i], t0, t1);
        v[2 * i] = __float_as_uint(p0) + (__float_as_uint(t0) << 23);      // the low bits of kRound are 0: n goes to the exponent
        v[2 * i + 1] = __float_as_uint(p1) + (__float_as_uint(t1) << 23);
    }
}
__device__ __forceinline__ uint32_t power(float y) {
    const Pair one[1] = {pair_of(y, y)};
    uint32_t v[2];
    power(one, v);
    return v[0];
}
__device__ __forceinline__ int bin_of(uint32_t v) {
    const int b = static_cast<int>(v >> kLowBits) - static_cast<int>(kFirstBits);
    return b < 0 ? kTail : b;
}
// Bits by which a weight of a bin is shifted to the left of its 24-bit mantissa.
__device__ __forceinline__ int shift_of_bin(int bin) {
    return static_cast<int>((static_cast<uint32_t>(bin) + kFirstBits) >> (23 - kLowBits)) - 150;
}
__device__ __forceinline__ unsigned long long weight_of(uint32_t v) {
    const int up = static_cast<int>(v >> 23) - 150;
    const uint32_t mantissa = (v & 0x7fffffu) | 0x800000u;
    return up >= 0 ? static_cast<unsigned long long>(mantissa) << up : up > -32 ? static_cast<unsigned long long>(mantissa >> -up) : 0ull;
}

// Exclusive prefixes of a weight and a number over the CTA in thread order, and the totals.
__device__ __forceinline__ Sums block_before(unsigned long long weight, uint32_t n, ScanSlots &slots, Sums &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long w = weight;
    uint32_t m = n;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const unsigned long long up = __shfl_up_sync(0xffffffffu, w, d);
        const uint32_t up_n = __shfl_up_sync(0xffffffffu, m, d);
        if (lane >= d) {
            w += up;
            m += up_n;
        }
    }
    __syncthreads();
    if (lane == 31) {
        slots.weight[warp] = w;
        slots.n[warp] = m;
    }
    __syncthreads();
    Sums before = {w - weight, m - n};
    total = {0, 0};
#pragma unroll
    for (int i = 0; i < kGivenWarps; ++i) {
        const unsigned long long x = slots.weight[i];
        const uint32_t y = slots.n[i];
        if (i < warp) {
            before.weight += x;
            before.n += y;
        }
        total.weight += x;
        total.n += y;
    }
    return before;
}

// floor(a b / 2^32) and whether something is left over, for a product of up to 96 bits.
__device__ __forceinline__ unsigned long long share_of(unsigned long long a, unsigned long long b, bool &rest) {
    const unsigned long long lo = a * b, hi = __umul64hi(a, b);
    rest = (lo & 0xffffffffull) != 0;
    return (hi << 32) | (lo >> 32);
}

// -0 becomes +0 and NaN becomes -inf, in every element.
template <int DTYPE>
__device__ __forceinline__ void settle(uint4 &w) {
    uint32_t *e = reinterpret_cast<uint32_t *>(&w);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DTYPE == SBW_DTYPE_F32) {
            e[i] = __float_as_uint(fmaxf(__fadd_rn(__uint_as_float(e[i]), 0.0f), -INFINITY));
        } else {
            const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162 *>(&e[i]);
            const __nv_bfloat162 zero = __floats2bfloat162_rn(0.0f, 0.0f), low = __floats2bfloat162_rn(-INFINITY, -INFINITY);
            const __nv_bfloat162 y = __hmax2(__hadd2(x, zero), low);
            e[i] = *reinterpret_cast<const uint32_t *>(&y);
        }
    }
}
// The infinite ones share everything: +inf becomes 0 and everything else -inf.
template <int DTYPE>
__device__ __forceinline__ void only_infinite(uint4 &w) {
    uint32_t *e = reinterpret_cast<uint32_t *>(&w);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DTYPE == SBW_DTYPE_F32) e[i] = e[i] == 0x7f800000u ? 0u : 0xff800000u;
        else e[i] = ((e[i] & 0xffffu) == 0x7f80u ? 0u : 0xff80u) | ((e[i] >> 16) == 0x7f80u ? 0u : 0xff800000u);
    }
}

// Where a CTA's dynamic shared memory begins.
[[maybe_unused]] __device__ __forceinline__ const void *room_base() {
    extern __shared__ __align__(16) uint8_t given_smem[];
    return given_smem;
}

// A CTA's part of a row.  Resident: its biased vectors are in shared memory after load().  Otherwise every pass reads
// them from global memory (the second time from L2) and biases them anew.
template <int DTYPE_, int SCHEME_, bool RESIDENT_>
struct Row {
    static constexpr int DTYPE = DTYPE_, SCHEME = SCHEME_;
    static constexpr bool RESIDENT = RESIDENT_;
    static constexpr int VEC = DTYPE == SBW_DTYPE_F32 ? 4 : 8;
    static_assert(!RESIDENT || DTYPE == SBW_DTYPE_F32, "");
    using Shared = GivenShared<RESIDENT ? 2 : kGivenWarps>;
    // loads in flight per thread
    static constexpr int kInFlight = SCHEME == kSchemeNone ? 4 : 2;

    const GivenArgs &a;
    int64_t row;
    const char *row_ptr, *base;   // its first element, and the 16-byte boundary at or before it
    uint32_t head;                // elements between the two
    uint32_t vec0, vectors;       // this CTA's vectors, counted from base
    uint32_t col0;                // column of their first element; columns before 0 wrap, their values are -inf
    uint32_t whole_from, wholes;  // those of the vectors that lie in the row with all their elements
    uint4 *slice;
    RowSeedS<SCHEME> rs;
    bool infinite;

    __device__ __forceinline__ Row(const GivenArgs &args, int64_t r, uint32_t part, uint4 *room)
        : a(args), row(r), slice(room), infinite(false) {
        row_ptr = static_cast<const char *>(a.logits) + row * a.ld * (16 / VEC);
        head = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row_ptr) % 16) / (16 / VEC);
        base = row_ptr - static_cast<int64_t>(head) * (16 / VEC);
        const uint32_t all = (head + static_cast<uint32_t>(a.V) + VEC - 1) / VEC;
        vec0 = min(part * a.part_vectors, all);
        vectors = min(a.part_vectors, all - vec0);
        col0 = vec0 * VEC - head;
        whole_from = vec0 == 0u && head ? 1u : 0u;
        const uint32_t end = (head + static_cast<uint32_t>(a.V)) / VEC;           // of the whole ones, counted from base
        wholes = min(vec0 + vectors, end) > vec0 + whole_from ? min(vec0 + vectors, end) - (vec0 + whole_from) : 0u;
        rs.init(a.bias.key, a.ctx + row * a.W, a.W);
    }
    __device__ __forceinline__ bool whole(uint32_t j) const { return j - whole_from < wholes; }
    __device__ __forceinline__ bool lies_here(const void *p, int n) const { return lies_in_rows(p, n, a.logits, 16 / VEC, a.B, a.V, a.ld); }
    __device__ __forceinline__ uint4 fetch(const uint4 *p) const {
        if (!SBW_CHECKED(lies_here(p, VEC), SBW_SITE_GIVEN_LOAD)) return make_uint4(0u, 0u, 0u, 0u);
        return __ldg(p);
    }
    __device__ __forceinline__ uint4 raw(uint32_t j) const { return fetch(reinterpret_cast<const uint4 *>(base) + vec0 + j); }
    // Vector j of a resident part.
    __device__ __forceinline__ uint4 kept(uint32_t j) const {
        if (!SBW_CHECKED(lies_in_shared(slice + j, 16, room_base()), SBW_SITE_GIVEN_SHARED)) return make_uint4(0u, 0u, 0u, 0u);
        return slice[j];
    }
    __device__ __forceinline__ void keep(uint32_t j, const uint4 &w) const {
        if (SBW_CHECKED(lies_in_shared(slice + j, 16, room_base()), SBW_SITE_GIVEN_SHARED)) slice[j] = w;
    }
    // The vector at an end of the row: what lies outside reads as -inf.  Biased.
    __device__ __forceinline__ uint4 ragged(uint32_t j) const {
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        uint32_t *e = reinterpret_cast<uint32_t *>(&w);
        const uint32_t col = col0 + j * VEC;
#pragma unroll 1
        for (int i = 0; i < VEC; ++i) {
            float x = -INFINITY;
            if (col + i < static_cast<uint32_t>(a.V) && SBW_CHECKED(lies_here(row_ptr + static_cast<int64_t>(col + i) * (16 / VEC), 1), SBW_SITE_GIVEN_LOAD))
                x = biased_at<DTYPE, SCHEME>(row_ptr, col + i, rs, a.vocab_offset + col + i, a.bias);
            if constexpr (DTYPE == SBW_DTYPE_F32) e[i] = __float_as_uint(x);
            else e[i >> 1] |= (i & 1) ? (__float_as_uint(x) & 0xffff0000u) : (__float_as_uint(x) >> 16);
        }
        return w;
    }
    // f(vector, j) for the thread's vectors from global memory, biased.  Whole batches of whole vectors need no checks.
    template <typename F>
    __device__ __forceinline__ void each_loaded(F f) const {
        const uint32_t end = whole_from + wholes;
        const uint4 *const from = reinterpret_cast<const uint4 *>(base) + vec0;
        const uint32_t vg = a.vocab_offset + col0;
        uint32_t j = whole_from + threadIdx.x;
        for (; j + (kInFlight - 1) * kGivenThreads < end; j += kInFlight * kGivenThreads) {
            uint4 w[kInFlight];
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) w[u] = fetch(from + j + u * kGivenThreads);
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) {
                bias_vector<DTYPE, SCHEME>(w[u], rs, vg + (j + u * kGivenThreads) * VEC, a.bias);
                f(w[u], j + u * kGivenThreads);
            }
        }
#pragma unroll 1
        for (; j < end; j += kGivenThreads) {
            uint4 w = fetch(from + j);
            bias_vector<DTYPE, SCHEME>(w, rs, vg + j * VEC, a.bias);
            f(w, j);
        }
        // the row's ragged ends
        if (threadIdx.x < 2u) {
            const uint32_t at = threadIdx.x == 0u ? 0u : vectors - 1u;
            if (vectors > threadIdx.x && !whole(at)) f(ragged(at), at);
        }
    }
    // f(vector, j) for the thread's vectors, biased.  Not settled where they come from global memory: NaN and -0 have the
    // weights that -inf and +0 have.
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        if constexpr (RESIDENT) {
            for (uint32_t j = threadIdx.x; j < vectors; j += kGivenThreads) f(kept(j), j);
        } else if (infinite) {
            for (uint32_t j = threadIdx.x; j < vectors; j += kGivenThreads) f(vector(j), j);
        } else {
            each_loaded(f);
        }
    }
    // One of them.
    __device__ __forceinline__ uint4 vector(uint32_t j) const {
        if constexpr (RESIDENT) return kept(j);
        uint4 w;
        if (whole(j)) {
            w = raw(j);
            bias_vector<DTYPE, SCHEME>(w, rs, a.vocab_offset + col0 + j * VEC, a.bias);
        } else {
            w = ragged(j);
        }
        settle<DTYPE>(w);
        if (infinite) only_infinite<DTYPE>(w);
        return w;
    }
    // Element i of vector j, which is one of the row's.
    __device__ __forceinline__ float value_at(uint32_t j, int i) const {
        float x;
        if constexpr (RESIDENT) {
            if (!SBW_CHECKED(lies_in_shared(slice + j, 16, room_base()), SBW_SITE_GIVEN_SHARED)) return -INFINITY;
            x = reinterpret_cast<const float *>(slice + j)[i];
        } else {
            const uint32_t col = col0 + j * VEC + i;
            if (!SBW_CHECKED(lies_here(row_ptr + static_cast<int64_t>(col) * (16 / VEC), 1), SBW_SITE_GIVEN_LOAD)) return -INFINITY;
            x = fmaxf(biased_at<DTYPE, SCHEME>(row_ptr, col, rs, a.vocab_offset + col, a.bias) + 0.0f, -INFINITY);
            if (infinite) x = x == INFINITY ? 0.0f : -INFINITY;
        }
        return x;
    }
    // Brings a resident part in; returns the thread's largest value.
    __device__ __forceinline__ float load() {
        float best = -INFINITY;
        each_loaded([&](uint4 w, uint32_t j) {
            settle<DTYPE>(w);
            if constexpr (RESIDENT) keep(j, w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) best = fmaxf(best, value(w, i));
        });
        return best;
    }
    __device__ __forceinline__ void keep_infinite() {
        infinite = true;
        if constexpr (RESIDENT)
            for (uint32_t j = threadIdx.x; j < vectors; j += kGivenThreads) {
                uint4 w = kept(j);
                only_infinite<DTYPE>(w);
                keep(j, w);
            }
    }
    static __device__ __forceinline__ float value(const uint4 &w, int i) {
        const uint32_t *e = reinterpret_cast<const uint32_t *>(&w);
        if constexpr (DTYPE == SBW_DTYPE_F32) return __uint_as_float(e[i]);
        else return __uint_as_float((i & 1) ? (e[i >> 1] & 0xffff0000u) : (e[i >> 1] << 16));
    }
    // Elements i and i + 1 of a vector.
    static __device__ __forceinline__ Pair values(const uint4 &w, int i) { return pair_of(value(w, i), value(w, i + 1)); }
};

__device__ __forceinline__ void count_one(uint32_t addr) {
    asm volatile("red.relaxed.cta.shared::cta.add.u32 [%0], %1;" ::"r"(addr), "r"(1u) : "memory");
}
// One candidate of weight u (fp32 bits; 0: none) in the histogram, at counters n and low, or its truncation `whole` to the
// tail.  Predicated: a branch per element would keep the elements of a vector from overlapping.
__device__ __forceinline__ void weigh_one(uint32_t u, uint32_t n, uint32_t low, uint32_t whole, uint32_t &tail) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ge.u32 p, %1, %2;\n\t"
                 "@p red.relaxed.cta.shared::cta.add.u32 [%3], 1;\n\t"
                 "@p red.relaxed.cta.shared::cta.add.u32 [%4], %5;\n\t"
                 "@!p add.u32 %0, %0, %6;\n\t}"
                 : "+r"(tail) : "r"(u), "r"(kFirstBits << kLowBits), "r"(n), "r"(low), "r"(u & ((1u << kLowBits) - 1u)), "r"(whole) : "memory");
}

template <typename ROW>
class Cluster {
  public:
    using Shared = typename ROW::Shared;
    Shared &sh;
    const ROW &row;
    const RowWeights rw;
    const uint32_t parts, part;
    static constexpr int kCopies = sizeof(Shared::hist.low) / sizeof(Shared::hist.low[0]);

    __device__ __forceinline__ Cluster(Shared &s, const ROW &r, const RowWeights &w, uint32_t n, uint32_t p)
        : sh(s), row(r), rw(w), parts(n), part(p) {}

    __device__ __forceinline__ void sync() const {
        if (parts > 1) cg::this_cluster().sync();
        else __syncthreads();
    }
    template <typename T>
    __device__ __forceinline__ T *at(T *p, uint32_t rank) const {
        return parts > 1 ? cg::this_cluster().map_shared_rank(p, rank) : p;
    }
    __device__ __forceinline__ uint32_t distance(float x) const { return rw.code_m - order_code(__float_as_uint(x)); }
    __device__ __forceinline__ unsigned long long weight_at(uint32_t dist) const {
        return weight_of(power(rw.log2_of(__uint_as_float(order_decode(rw.code_m - dist)))));
    }
    __device__ __forceinline__ Pair log2_of(Pair x) const {
        return pair_mul(pair_add(x, pair_of(-rw.m, -rw.m)), pair_of(rw.c, rw.c));
    }

    // The CTA's candidates in bins, those of the tail summed.  No branch, so that the elements of a vector overlap.
    __device__ __forceinline__ void histogram() const {
        uint32_t *const all = reinterpret_cast<uint32_t *>(&sh.hist);
        for (int i = threadIdx.x; i < static_cast<int>(sizeof(sh.hist) / 4); i += kGivenThreads) all[i] = 0u;
        __syncthreads();
        // addresses less what the first bin's bits come to
        const uint32_t at_n = static_cast<uint32_t>(__cvta_generic_to_shared(sh.hist.n)) - 4u * kFirstBits;
        const uint32_t at_low = static_cast<uint32_t>(__cvta_generic_to_shared(sh.hist.low[(threadIdx.x >> 5) % kCopies])) - 4u * kFirstBits;
        unsigned long long tail = 0;
        uint32_t number = 0;                             // of all candidates
        row.each([&](const uint4 &w, uint32_t) {
            constexpr int VEC = ROW::VEC;
            uint32_t some = 0;                           // of 8 weights of 25 bits
            Pair y[VEC / 2];
            uint32_t v[VEC];
#pragma unroll
            for (int i = 0; i < VEC / 2; ++i) y[i] = log2_of(ROW::values(w, 2 * i));
            power(y, v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float yy[2];
                of_pair(y[i / 2], yy[0], yy[1]);
                const bool real = yy[i & 1] >= rw.lowest;
                uint32_t u = real ? v[i] : 0u;
                number += real;
                if (!SBW_CHECKED(u < (kFirstBits << kLowBits) || (u >> kLowBits) - kFirstBits < kBins, SBW_SITE_GIVEN_SHARED)) u = 0u;
                weigh_one(u, at_n + 4u * (u >> kLowBits), at_low + 4u * (u >> kLowBits), __float2uint_rz(__uint_as_float(u)), some);
            }
            tail += some;
        });
        Sums total;
        block_before(tail, number, sh.scan, total);      // its barriers also end the histogram
        // the bins' weights
        uint32_t binned = 0;
#pragma unroll
        for (int k = 0; k < kBins / kGivenThreads; ++k) {
            const uint32_t bin = k * kGivenThreads + threadIdx.x, n = sh.hist.n[bin], v = (bin + kFirstBits) << kLowBits;
            unsigned long long low = static_cast<unsigned long long>(n) * ((v & 0x7fffffu) | 0x800000u);
#pragma unroll
            for (int q = 0; q < kCopies; ++q) low += sh.hist.low[q][bin];
            sh.bins.n[bin] = n;
            sh.bins.weight[bin] = low << shift_of_bin(static_cast<int>(bin));
            binned += n;
        }
        Sums total_binned;
        block_before(0ull, binned, sh.scan, total_binned);
        if (threadIdx.x == 0) {
            at(sh.tail_weight, 0)[part] = total.weight;
            at(sh.tail_n, 0)[part] = total.n - total_binned.n;
        }
    }

    // Every CTA adds up a share of the bins over all CTAs, in the first one's place: nobody else touches them.
    __device__ __forceinline__ void merge() const {
        sync();
        if (parts == 1) return;
        const uint32_t share = kBins / parts;            // a power of two, at most one bin per thread
        if (threadIdx.x < share) {
            const uint32_t bin = part * share + threadIdx.x;
            uint32_t n = 0;
            unsigned long long w = 0;
#pragma unroll
            for (uint32_t r = 0; r < kMaxParts; ++r) {       // unrolled: the loads from other SMs overlap
                if (r >= parts) break;
                n += *at(&sh.bins.n[bin], r);
                w += *at(&sh.bins.weight[bin], r);
            }
            *at(&sh.bins.n[bin], 0) = n;
            *at(&sh.bins.weight[bin], 0) = w;
        }
        sync();
    }

    // f(column, weight's bits, distance) for the candidates that a command names.
    template <typename F>
    __device__ __forceinline__ void each_named(const Command &c, F f) const {
        constexpr int VEC = ROW::VEC;
        // log2 of the bins' ends, with a margin for the rounding of y and of the logarithm
        const float from = c.bin_lo == kTail ? rw.lowest
                                             : fmaxf(rw.lowest, __log2f(__uint_as_float((c.bin_lo + kFirstBits) << kLowBits)) - 40.001f);
        const float to = __log2f(__uint_as_float((c.bin_hi + 1 + kFirstBits) << kLowBits)) - 39.999f;
        row.each([&](const uint4 &w, uint32_t j) {
            uint32_t hits = 0;
#pragma unroll
            for (int i = 0; i < VEC; i += 2) {
                float y0, y1;
                of_pair(log2_of(ROW::values(w, i)), y0, y1);
                if (y0 >= from && y0 <= to) hits |= 1u << i;
                if (y1 >= from && y1 <= to) hits |= 2u << i;
            }
            // few: their values are fetched again, which keeps this loop's body small
#pragma unroll 1
            while (hits) {
                const int i = __ffs(hits) - 1;
                hits &= hits - 1u;
                const float x = row.value_at(j, i);
                const uint32_t v = power(rw.log2_of(x)), dist = distance(x);
                const int bin = bin_of(v);
                if (bin >= c.bin_lo && bin <= c.bin_hi && dist >= c.dist_lo && dist <= c.dist_hi) f(row.col0 + j * VEC + i, v, dist);
            }
        });
    }

    __device__ __forceinline__ void obey(const Command &c) const {
        if (c.op == kGather) {
            // into the CTA's own list first: an add to another SM's counter takes a microsecond to answer
            if (part != 0) {
                if (threadIdx.x == 0) sh.list_n = 0u;
                __syncthreads();
            }
            each_named(c, [&](uint32_t col, uint32_t, uint32_t dist) {
                const uint32_t i = atomicAdd(&sh.list_n, 1u);
                (void)SBW_CHECKED(i < kListCap, SBW_SITE_GIVEN_SHARED);      // a list is asked for where it holds all
                if (i < kListCap) sh.list[i] = static_cast<unsigned long long>(dist) << 32 | col;
            });
            if (part != 0) {
                __syncthreads();
                const uint32_t n = min(sh.list_n, static_cast<uint32_t>(kListCap));
                if (n == 0u) return;
                if (threadIdx.x == 0) sh.list_at = atomicAdd(at(&sh.list_n, 0), n);
                __syncthreads();
                const uint32_t first = sh.list_at;
                unsigned long long *const list = at(sh.list, 0);
                for (uint32_t i = threadIdx.x; i < n; i += kGivenThreads)
                    if (SBW_CHECKED(first + i < kListCap, SBW_SITE_GIVEN_SHARED) && first + i < kListCap) list[first + i] = sh.list[i];
            }
        } else if (c.op == kSplit) {
            if (part != 0) {                             // the first CTA has cleared its own
                for (int i = threadIdx.x; i < kFine; i += kGivenThreads) sh.fine.n[i] = sh.fine.lo[i] = sh.fine.hi[i] = 0u;
                __syncthreads();
            }
            each_named(c, [&](uint32_t, uint32_t v, uint32_t dist) {
                const uint32_t bin = (dist - c.dist_lo) >> c.shift;
                if (!SBW_CHECKED(bin < kFine, SBW_SITE_GIVEN_SHARED)) return;
                // of a bin the mantissa (the exponent is the bin's), of the tail the weight itself
                const uint32_t q = c.bin_lo == kTail ? static_cast<uint32_t>(weight_of(v)) : (v & 0x7fffffu) | 0x800000u;
                atomicAdd(&sh.fine.n[bin], 1u);
                atomicAdd(&sh.fine.lo[bin], q & ((1u << kLimb) - 1u));
                atomicAdd(&sh.fine.hi[bin], q >> kLimb);
            });
            if (part != 0) {
                __syncthreads();
                for (int i = threadIdx.x; i < kFine; i += kGivenThreads) {
                    if (sh.fine.n[i] == 0u) continue;
                    atomicAdd(at(&sh.fine.n[i], 0), sh.fine.n[i]);
                    atomicAdd(at(&sh.fine.lo[i], 0), sh.fine.lo[i]);
                    atomicAdd(at(&sh.fine.hi[i], 0), sh.fine.hi[i]);
                }
            }
        } else {
            // candidates of one value, in the order of their columns: a run of vectors per thread
            constexpr int VEC = ROW::VEC;
            const float x = __uint_as_float(order_decode(rw.code_m - c.dist_lo));
            const uint32_t run = (row.vectors + kGivenThreads - 1) / kGivenThreads;
            const uint32_t begin = min(threadIdx.x * run, row.vectors), end = min(begin + run, row.vectors);
            uint32_t mine = 0;
            for (uint32_t j = begin; j < end; ++j) {
                const uint4 w = row.vector(j);
#pragma unroll
                for (int i = 0; i < VEC; ++i) mine += ROW::value(w, i) == x;
            }
            Sums total;
            const uint32_t before = block_before(0ull, mine, sh.scan, total).n;
            if (c.op == kCountTies) {
                if (threadIdx.x == 0) at(sh.ties, 0)[part] = total.n;
            } else if (c.part == part && before <= c.which && c.which < before + mine) {
                uint32_t left = c.which - before;
                for (uint32_t j = begin; j < end; ++j) {
                    const uint4 w = row.vector(j);
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        if (ROW::value(w, i) == x && left-- == 0u) *at(&sh.tie_col, 0) = row.col0 + j * VEC + i;
                }
            }
        }
    }

    // First CTA: has everyone obey, itself too.
    __device__ __forceinline__ void order(const Command &c) const {
        if (threadIdx.x < parts) *at(&sh.cmd, threadIdx.x) = c;
        sync();
        if (c.op == kDone) return;
        obey(c);
        sync();
    }
    __device__ __forceinline__ void serve() const {
        for (;;) {
            sync();
            const Command c = sh.cmd;
            if (c.op == kDone) return;
            obey(c);
            sync();
        }
    }
};

// The answer to one question: the candidate, and the running number and weight up to and with it.
struct Found {
    uint32_t dist, col, n;
    unsigned long long running, own;
};

// First CTA: the row's bins, scanned, and the list that was made last.
template <typename ROW>
class Finder {
    static constexpr int kOwn = kBins / kGivenThreads, kOwnFine = kFine / kGivenThreads, kOwnList = kListCap / kGivenThreads;
    const Cluster<ROW> &cl;
    typename ROW::Shared &sh;
    uint32_t own_n0;                       // before this thread's bins (which run from the last down)
    unsigned long long own_w0;
    uint32_t bins_n;                       // of all bins but the tail
    unsigned long long bins_w;
    // the list: what comes before it, what it holds
    uint32_t list_n0 = 0, list_n = 0;
    unsigned long long list_w0 = 0, list_w = 0;
    unsigned long long item_w[kOwnList], items_w0;

  public:
    uint32_t total_n;
    unsigned long long total_w;

    __device__ __forceinline__ explicit Finder(const Cluster<ROW> &c) : cl(c), sh(c.sh) {
        unsigned long long w = 0;
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            w += sh.bins.weight[kBins - 1 - (threadIdx.x * kOwn + i)];
            n += sh.bins.n[kBins - 1 - (threadIdx.x * kOwn + i)];
        }
        Sums all;
        const Sums before = block_before(w, n, sh.scan, all);
        own_w0 = before.weight;
        own_n0 = before.n;
        bins_w = all.weight;
        bins_n = all.n;
        total_n = bins_n;
        total_w = bins_w;
        for (uint32_t r = 0; r < cl.parts; ++r) {
            total_n += sh.tail_n[r];
            total_w += sh.tail_weight[r];
        }
    }

    // The first candidate at which the running number (by_weight false) or weight reaches target, 1 .. the total.
    __device__ __forceinline__ Found find(bool by_weight, unsigned long long target) {
        const bool listed = by_weight ? target > list_w0 && target <= list_w0 + list_w
                                      : target > list_n0 && target <= static_cast<unsigned long long>(list_n0) + list_n;
        if (!listed) {
            Found tie;
            if (fetch(by_weight, target, tie)) return tie;
        }
        return walk(by_weight, target);
    }

  private:
    __device__ __forceinline__ void found_bin(int at, uint32_t n_before, uint32_t n, unsigned long long w_before, unsigned long long w) {
        sh.found_at = at;
        sh.found_n_before = n_before;
        sh.found_n = n;
        sh.found_before = w_before;
        sh.found_weight = w;
    }

    // Makes a list that holds the candidate; true if it was found on the way, as one of many equal ones.
    __device__ __forceinline__ bool fetch(bool by_weight, unsigned long long target, Found &tie) {
        __syncthreads();
        if (threadIdx.x == 0) found_bin(kTail, bins_n, total_n - bins_n, bins_w, total_w - bins_w);
        __syncthreads();
        {
            uint32_t n = own_n0;
            unsigned long long w = own_w0;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const int bin = kBins - 1 - static_cast<int>(threadIdx.x * kOwn + i);
                const uint32_t bn = sh.bins.n[bin];
                const unsigned long long bw = sh.bins.weight[bin];
                if (by_weight ? w < target && w + bw >= target : n < target && n + bn >= target) found_bin(bin, n, bn, w, bw);
                n += bn;
                w += bw;
            }
        }
        __syncthreads();
        Command c = {};
        c.op = kGather;
        c.bin_lo = c.bin_hi = sh.found_at;
        c.dist_lo = 0u;
        c.dist_hi = 0xffffffffu;
        list_n0 = sh.found_n_before;
        list_w0 = sh.found_before;
        uint32_t number = sh.found_n;
        if (list_n0 + number <= kPrefixCap) {            // everything from the first candidate on
            c.bin_hi = kBins - 1;
            number += list_n0;
            list_n0 = 0u;
            list_w0 = 0ull;
        }
        uint32_t bits = 32;
        while (number > kListCap) {
            // too many: by distance, ten bits at a time
            if (bits == 0) {
                tie = pick(by_weight, target, c, number);
                return true;
            }
            __syncthreads();
            for (int i = threadIdx.x; i < kFine; i += kGivenThreads) sh.fine.n[i] = sh.fine.lo[i] = sh.fine.hi[i] = 0u;
            list_n = 0u;
            list_w = 0ull;
            const uint32_t shift = bits > 10 ? bits - 10 : 0;
            c.op = kSplit;
            c.shift = shift;
            cl.order(c);
            const int up = c.bin_lo == kTail ? 0 : shift_of_bin(c.bin_lo);      // weights of the tail are held as they are
            unsigned long long w[kOwnFine], sum_w = 0;
            uint32_t n[kOwnFine], sum_n = 0;
#pragma unroll
            for (int i = 0; i < kOwnFine; ++i) {
                const int bin = threadIdx.x * kOwnFine + i;
                n[i] = sh.fine.n[bin];
                w[i] = (static_cast<unsigned long long>(sh.fine.lo[bin]) + (static_cast<unsigned long long>(sh.fine.hi[bin]) << kLimb)) << up;
                sum_n += n[i];
                sum_w += w[i];
            }
            Sums all;
            const Sums before = block_before(sum_w, sum_n, sh.scan, all);
            unsigned long long wb = list_w0 + before.weight;
            uint32_t nb = list_n0 + before.n;
#pragma unroll
            for (int i = 0; i < kOwnFine; ++i) {
                if (by_weight ? wb < target && wb + w[i] >= target : nb < target && nb + n[i] >= target)
                    found_bin(static_cast<int>(threadIdx.x) * kOwnFine + i, nb, n[i], wb, w[i]);
                nb += n[i];
                wb += w[i];
            }
            __syncthreads();
            c.dist_lo += static_cast<uint32_t>(sh.found_at) << shift;
            c.dist_hi = c.dist_lo + ((1u << shift) - 1u);
            list_n0 = sh.found_n_before;
            list_w0 = sh.found_before;
            number = sh.found_n;
            bits = shift;
        }
        __syncthreads();
        if (threadIdx.x == 0) sh.list_n = 0u;
        c.op = kGather;
        cl.order(c);
        list_n = min(sh.list_n, static_cast<uint32_t>(kListCap));
        sort();
        unsigned long long sum = 0;
#pragma unroll
        for (int i = 0; i < kOwnList; ++i) {
            const uint32_t j = threadIdx.x * kOwnList + i;
            item_w[i] = j < list_n ? cl.weight_at(static_cast<uint32_t>(sh.list[j] >> 32)) : 0ull;
            sum += item_w[i];
        }
        Sums all;
        items_w0 = block_before(sum, 0u, sh.scan, all).weight;
        list_w = all.weight;
        return false;
    }

    // One of `number` candidates of the same value, those of the command's distance.
    __device__ __forceinline__ Found pick(bool by_weight, unsigned long long target, Command c, uint32_t number) {
        Found r;
        r.dist = c.dist_lo;
        r.own = cl.weight_at(c.dist_lo);
        const unsigned long long j = by_weight ? (target - list_w0 + r.own - 1) / r.own : target - list_n0;     // from 1 on
        c.op = kCountTies;
        cl.order(c);
        uint32_t before = 0, p = 0;
        while (p + 1 < cl.parts && j > before + sh.ties[p]) before += sh.ties[p++];
        c.op = kPickTie;
        c.part = p;
        c.which = static_cast<uint32_t>(j - 1) - before;
        __syncthreads();
        cl.order(c);
        r.col = sh.tie_col;
        r.n = list_n0 + static_cast<uint32_t>(j);
        r.running = list_w0 + j * r.own;
        list_n = 0u;                                     // no list is left
        list_w = 0ull;
        return r;
    }

    // Ascending: a short list by counting the smaller ones, else bitonic.
    __device__ __forceinline__ void sort() {
        if (list_n <= kCountingSort) {
            const unsigned long long mine = threadIdx.x < list_n ? sh.list[threadIdx.x] : 0ull;
            uint32_t rank = 0;
            if (threadIdx.x < list_n) {
#pragma unroll 8
                for (uint32_t i = 0; i < list_n; ++i) rank += sh.list[i] < mine;
            }
            __syncthreads();
            if (threadIdx.x < list_n && SBW_CHECKED(rank < list_n, SBW_SITE_GIVEN_SHARED)) sh.list[rank] = mine;
            __syncthreads();
            return;
        }
        uint32_t len = 2;
        while (len < list_n) len <<= 1;
        for (uint32_t i = list_n + threadIdx.x; i < len; i += kGivenThreads) sh.list[i] = ~0ull;
        __syncthreads();
        for (uint32_t k = 2; k <= len; k <<= 1) {
            for (uint32_t j = k >> 1; j > 0; j >>= 1) {
                for (uint32_t t = threadIdx.x; t < len / 2; t += kGivenThreads) {
                    const uint32_t i = ((t & ~(j - 1)) << 1) | (t & (j - 1));
                    if (!SBW_CHECKED(i + j < kListCap, SBW_SITE_GIVEN_SHARED)) continue;
                    const unsigned long long x = sh.list[i], y = sh.list[i + j];
                    if ((x > y) == ((i & k) == 0)) {
                        sh.list[i] = y;
                        sh.list[i + j] = x;
                    }
                }
                __syncthreads();
            }
        }
    }

    __device__ __forceinline__ Found walk(bool by_weight, unsigned long long target) {
        __syncthreads();
        unsigned long long w = list_w0 + items_w0;
#pragma unroll
        for (int i = 0; i < kOwnList; ++i) {
            const uint32_t j = threadIdx.x * kOwnList + i;
            if (j < list_n && (by_weight ? w < target && w + item_w[i] >= target : list_n0 + j + 1u == target)) {
                found_bin(static_cast<int>(j), 0u, 0u, w, item_w[i]);
                sh.found_dist = static_cast<uint32_t>(sh.list[j] >> 32);
                sh.found_col = static_cast<uint32_t>(sh.list[j]);
            }
            w += item_w[i];
        }
        __syncthreads();
        return Found{sh.found_dist, sh.found_col, list_n0 + static_cast<uint32_t>(sh.found_at) + 1u, sh.found_before + sh.found_weight, sh.found_weight};
    }
};

// ---- a row by its weights -------------------------------------------------------------------

// The three questions in turn: ask(by_weight, target) finds the candidate at which the running number or weight reaches
// the target; the first two leave the running number and weight up to it.  The last answer is what is drawn.
template <typename F>
__device__ __forceinline__ void narrow(const Settings &set, uint32_t &kept, unsigned long long &total, F ask) {
#pragma unroll 1
    for (int question = 0; question < 3; ++question) {
        bool rest;
        unsigned long long target;
        if (question == 0) {
            if (set.top_k <= 0 || set.top_k >= kept) continue;
            target = static_cast<unsigned long long>(set.top_k);
        } else if (question == 1) {
            if (!set.p32) continue;
            target = share_of(set.p32, total, rest);
            target += rest;
            if (target >= total) continue;
        } else {
            target = share_of(set.u32, total, rest) + 1ull;
        }
        uint32_t n;
        unsigned long long w;
        ask(question != 0, target, n, w);
        if (question < 2) {
            kept = n;
            total = w;
        }
    }
}

__device__ __forceinline__ void put_token(const GivenArgs &a, int64_t row, uint32_t col) {
    if (SBW_CHECKED(row >= 0 && row < a.B && col < a.V, SBW_SITE_GIVEN_OUTPUT)) a.out_tokens[row] = static_cast<int32_t>(col);
}
__device__ __forceinline__ void answer(const GivenArgs &a, int64_t row, uint32_t kept, unsigned long long own, unsigned long long total) {
    if (!SBW_CHECKED(row >= 0 && row < a.B, SBW_SITE_GIVEN_OUTPUT)) return;
    if (a.out_prob) a.out_prob[row] = total ? static_cast<float>(static_cast<double>(own) / static_cast<double>(total)) : 0.0f;
    if (a.out_kept) a.out_kept[row] = static_cast<int32_t>(kept);
}

// The whole of a row whose CTAs have all begun.
template <typename ROW>
__device__ __forceinline__ void by_weights(const GivenArgs &a, int64_t row, uint32_t part, uint8_t *smem) {
    auto &sh = *reinterpret_cast<typename ROW::Shared *>(smem);
    constexpr size_t kShared = (sizeof(typename ROW::Shared) + 15) / 16 * 16;
    ROW r(a, row, part, reinterpret_cast<uint4 *>(smem + kShared));
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (part == 0 && warp == kGivenWarps - 1) {
        const Settings set(a, row);
        for (uint32_t i = lane; i < a.parts; i += 32) *(a.parts > 1 ? cg::this_cluster().map_shared_rank(&sh.set, i) : &sh.set) = set;
    }
    float m = r.load();
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    if (lane == 0) sh.warp_max[warp] = m;
    __syncthreads();
    for (int w = 0; w < kGivenWarps; ++w) m = fmaxf(m, sh.warp_max[w]);
    if (a.parts > 1) {
        if (threadIdx.x < a.parts) cg::this_cluster().map_shared_rank(sh.part_max, threadIdx.x)[part] = m;
        cg::this_cluster().sync();
        for (uint32_t i = 0; i < a.parts; ++i) m = fmaxf(m, sh.part_max[i]);
    }
    if (m == -INFINITY) {                                // nothing can be drawn: every CTA of the cluster sees it
        if (part == 0 && threadIdx.x == 0) {
            put_token(a, r.row, 0u);
            answer(a, r.row, 0u, 0ull, 0ull);
        }
        return;
    }
    if (m == INFINITY) {
        r.keep_infinite();
        __syncthreads();
        m = 0.0f;
    }
    const Settings set = sh.set;
    RowWeights rw;
    rw.m = m;
    rw.code_m = order_code(__float_as_uint(m));
    rw.c = set.c;
    rw.lowest = set.lowest;
    const Cluster<ROW> cl(sh, r, rw, a.parts, part);
    cl.histogram();
    cl.merge();
    if (part != 0) {
        cl.serve();
        return;
    }
    Finder<ROW> finder(cl);
    uint32_t kept = finder.total_n;
    unsigned long long total = finder.total_w;
    Found f;
    narrow(set, kept, total, [&](bool by_weight, unsigned long long t, uint32_t &n, unsigned long long &w) {
        f = finder.find(by_weight, t);
        n = f.n;
        w = f.running;
    });
    if (threadIdx.x == 0) {
        put_token(a, r.row, f.col);
        answer(a, r.row, kept, f.own, total);
    }
    Command done = {};
    cl.order(done);
}

// fp32 rows.  Plain ones are read again by every pass, a CTA per row if there are as many rows as SMs (256 x 151936: 111 us;
// 330 with the row resident in the shared memory of a cluster, which then waits for its first CTA).
template <int DTYPE, int SCHEME>
using RowOf = Row<DTYPE, SCHEME, SCHEME != kSchemeNone>;
template <int DTYPE, int SCHEME>
__global__ void __launch_bounds__(kGivenThreads, SCHEME == kSchemeNone ? 2 : 1) given_kernel(const GivenArgs a) {
    using R = RowOf<DTYPE, SCHEME>;
    extern __shared__ __align__(16) uint8_t given_smem[];
    if (a.parts > 1) cg::this_cluster().sync();          // every CTA has begun: its shared memory can be written
    by_weights<R>(a, blockIdx.x / a.parts, blockIdx.x % a.parts, given_smem);
}

// Out of line, so that what it holds does not weigh on the kernel that hardly ever calls it.
template <typename ROW>
__device__ __noinline__ void by_weights_rare(const GivenArgs &a, int64_t row, uint32_t part, uint8_t *smem) {
    by_weights<ROW>(a, row, part, smem);
}

// ---- bf16: a row by its values --------------------------------------------------------------

// A bf16 row has few distinct values, so candidates are counted by value: one pass over the row, before its maximum is
// known, and one add per element; everything else happens on the counters.  The counters are the values of magnitude
// 2^-56 to 256, of either sign; the ends stand for what lies beyond them as well, zero included (so low a magnitude
// leaves the differences from the maximum and so the weights as zero does, unless the maximum is about as small).  Rows
// with a value from 256 on, rows in which values from -256 down have a weight, rows with a maximum below 2^-20 and rows
// whose token is one of several different values around zero are done by their weights instead.  A second pass finds the
// column of the value that was drawn.
constexpr uint32_t kCodes = 8192;                        // magnitudes per sign
constexpr uint32_t kFirstCode = (71u << 7) + 1u;         // the bits of the smallest magnitude, which is 2^-56 (1 + 2^-7)
static_assert(2 * kCodes == 32 * kGivenThreads, "a thread per block of 32 places");
static_assert(2 * kCodes * 4 == 1 << 16, "an offset of 16 bits stays within the counters");
struct CodesShared {
    uint32_t n[2 * kCodes];                              // positive ones by magnitude, then negative ones
    unsigned long long block_weight[2 * kCodes / 32];    // of 32 places
    uint32_t block_n[2 * kCodes / 32];
    uint32_t warp_best[kGivenWarps], part_best[kMaxParts];
    Settings set;
    ScanSlots scan;
    // what the first CTA tells the others
    uint32_t by_weights, value, which, around_zero;
    uint32_t tiny;                                       // some value around zero is not zero
    // a question
    unsigned long long weight_before, running, own;
    uint32_t block, n_before, found_n, found_value, found_which, found_all;
    uint32_t warp_ties[kGivenWarps], part_ties[kMaxParts];
};

// In the order of candidates the positive values come first, in blocks of 32 places.  Bits of the fp32 value of place o
// (zero for the smallest of either sign), and its counter.
__device__ __forceinline__ uint32_t value_of_place(uint32_t o) {
    return o - (kCodes - 1) < 2u ? 0u : (o < kCodes ? kFirstCode + (kCodes - 1 - o) : 0x8000u + kFirstCode + (o - kCodes)) << 16;
}
__device__ __forceinline__ uint32_t counter_of_place(uint32_t o) { return o < kCodes ? kCodes - 1 - o : o; }

template <int SCHEME>
__global__ void __launch_bounds__(kGivenThreads, SCHEME == kSchemeNone ? 2 : 1) given_codes_kernel(const GivenArgs a) {
    using R = Row<SBW_DTYPE_BF16, SCHEME, false>;
    extern __shared__ __align__(16) uint8_t given_smem[];
    CodesShared &sh = *reinterpret_cast<CodesShared *>(given_smem);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t part = blockIdx.x % a.parts;
    R r(a, blockIdx.x / a.parts, part, nullptr);
    const auto sync = [&] {
        if (a.parts > 1) cg::this_cluster().sync();
        else __syncthreads();
    };
    for (uint32_t i = threadIdx.x; i < 2 * kCodes / 4; i += kGivenThreads) reinterpret_cast<uint4 *>(sh.n)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (threadIdx.x == 0) sh.tiny = 0u;
    __syncthreads();
    // the settings take fp64 divisions and a logarithm: one warp's time, beside the others' loads
    if (part == 0 && warp == kGivenWarps - 1) {
        const Settings set(a, r.row);
        if (lane == 0) sh.set = set;
    }

    __nv_bfloat162 largest = __floats2bfloat162_rn(-256.0f, -256.0f);
    const __nv_bfloat162 smallest = __halves2bfloat162(__ushort_as_bfloat16(kFirstCode), __ushort_as_bfloat16(kFirstCode));
    const uint32_t counters = static_cast<uint32_t>(__cvta_generic_to_shared(sh.n));
    r.each_loaded([&](const uint4 &w, uint32_t) {
        const uint32_t *e = reinterpret_cast<const uint32_t *>(&w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // two values at a time: NaN and what is below -256 to -256, magnitudes to the counters' range
            const __nv_bfloat162 x = __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&e[i]), __floats2bfloat162_rn(-256.0f, -256.0f));
            const __nv_bfloat162 size = __hmin2(__hmax2(__habs2(x), smallest), __floats2bfloat162_rn(256.0f, 256.0f));
            largest = __hmax2(largest, x);
            // 13 bits of magnitude and the sign above them, twice, as offsets in bytes
            const uint32_t both = ((*reinterpret_cast<const uint32_t *>(&size) - kFirstCode * 0x10001u) |
                                   (*reinterpret_cast<const uint32_t *>(&x) >> 2 & 0x20002000u)) << 2;
            count_one(counters + (both & 0xffffu));
            count_one(counters + (both >> 16));
        }
    });
    // order code of the largest value (-0 counts as +0)
    uint32_t best = order_code(__float_as_uint(fmaxf(__low2float(largest), __high2float(largest)) + 0.0f));
    best = __reduce_max_sync(0xffffffffu, best);
    if (lane == 0) sh.warp_best[warp] = best;
    sync();
    if (a.parts > 1) {
        // a CTA adds up a share of the counters over all CTAs, in the first one's place: nobody else touches them
        const uint32_t share = 2 * kCodes / a.parts;     // 4 counters for each of a thread's trips
        uint4 *const first = reinterpret_cast<uint4 *>(cg::this_cluster().map_shared_rank(sh.n, 0) + part * share);
        for (uint32_t i = threadIdx.x; i < share / 4; i += kGivenThreads) {
            uint4 n = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (uint32_t q = 0; q < kMaxParts; ++q) {
                if (q >= a.parts) break;
                const uint4 x = reinterpret_cast<const uint4 *>(cg::this_cluster().map_shared_rank(sh.n, q) + part * share)[i];
                n.x += x.x;
                n.y += x.y;
                n.z += x.z;
                n.w += x.w;
            }
            first[i] = n;
        }
        if (threadIdx.x < kGivenWarps) {
            best = __reduce_max_sync((1u << kGivenWarps) - 1u, sh.warp_best[threadIdx.x]);
            if (threadIdx.x == 0) {
                cg::this_cluster().map_shared_rank(sh.part_best, 0)[part] = best;
            }
        }
        cg::this_cluster().sync();
    }

    if (part == 0) {
        const Settings set = sh.set;
        if (a.parts > 1) {
            for (uint32_t i = 0; i < a.parts; ++i) best = max(best, sh.part_best[i]);
        } else {
            for (int i = 0; i < kGivenWarps; ++i) best = max(best, sh.warp_best[i]);
        }
        RowWeights rw;
        rw.m = __uint_as_float(order_decode(best));
        rw.c = set.c;
        rw.lowest = set.lowest;
        // values beyond the counters that matter
        const bool beyond = rw.m >= 256.0f || fabsf(rw.m) < 0x1p-20f || rw.m <= -256.0f ||
                            (sh.n[2 * kCodes - 1] != 0u && rw.log2_of(-256.0f) >= rw.lowest);
        if (beyond) {
            if (threadIdx.x < a.parts) {
                uint32_t *const flag = &sh.by_weights;
                *(a.parts > 1 ? cg::this_cluster().map_shared_rank(flag, threadIdx.x) : flag) = 1u;
            }
        } else {
            const auto weight = [&](uint32_t value) -> unsigned long long {
                const float y = rw.log2_of(__uint_as_float(value));
                return y >= rw.lowest ? weight_of(power(y)) : 0ull;
            };
            // weights of the blocks, a warp per block and a lane per value
            uint32_t some = 0;                           // which of the warp's 32 have candidates
#pragma unroll 8
            for (int i = 0; i < 32; ++i) {
                const bool any = __any_sync(0xffffffffu, sh.n[counter_of_place((i * kGivenWarps + warp) * 32 + lane)] != 0u);
                some |= static_cast<uint32_t>(any) << i;
            }
            sh.block_weight[lane * kGivenWarps + warp] = 0ull;
            sh.block_n[lane * kGivenWarps + warp] = 0u;
            __syncwarp();
#pragma unroll 1
            while (some) {
                const uint32_t block = (__ffs(some) - 1) * kGivenWarps + warp;
                some &= some - 1u;
                const uint32_t num = sh.n[counter_of_place(block * 32 + lane)];
                unsigned long long w = weight(value_of_place(block * 32 + lane));
                const uint32_t n = __reduce_add_sync(0xffffffffu, w ? num : 0u);
                w *= num;                                // below 2^60: three sums of 20 bits
                w = __reduce_add_sync(0xffffffffu, static_cast<uint32_t>(w) & 0xfffffu) +
                    (static_cast<unsigned long long>(__reduce_add_sync(0xffffffffu, static_cast<uint32_t>(w >> 20) & 0xfffffu)) << 20) +
                    (static_cast<unsigned long long>(__reduce_add_sync(0xffffffffu, static_cast<uint32_t>(w >> 40))) << 40);
                if (lane == 0) {
                    sh.block_weight[block] = w;
                    sh.block_n[block] = n;
                }
            }
            __syncthreads();
            const unsigned long long sum_w = sh.block_weight[threadIdx.x];
            const uint32_t sum_n = sh.block_n[threadIdx.x];
            Sums all;
            const Sums before = block_before(sum_w, sum_n, sh.scan, all);
            // the value at which a target is reached: its block, then a lane per value
            const auto find = [&](bool by_weight, unsigned long long target, uint32_t &found_n, unsigned long long &running) {
                if (by_weight ? before.weight < target && target <= before.weight + sum_w
                              : before.n < target && target <= before.n + static_cast<unsigned long long>(sum_n)) {
                    sh.block = threadIdx.x;
                    sh.weight_before = before.weight;
                    sh.n_before = before.n;
                }
                __syncthreads();
                if (warp == 0) {
                    const uint32_t place = (SBW_CHECKED(sh.block < 2 * kCodes / 32, SBW_SITE_GIVEN_SHARED) ? sh.block : 0u) * 32 + lane;
                    const uint32_t value = value_of_place(place);
                    const unsigned long long w = weight(value);
                    const uint32_t num = w ? sh.n[counter_of_place(place)] : 0u;
                    unsigned long long w_to = w * num;
                    uint32_t n_to = num;
#pragma unroll
                    for (int d = 1; d < 32; d <<= 1) {
                        const unsigned long long up = __shfl_up_sync(0xffffffffu, w_to, d);
                        const uint32_t up_n = __shfl_up_sync(0xffffffffu, n_to, d);
                        if (lane >= d) {
                            w_to += up;
                            n_to += up_n;
                        }
                    }
                    w_to += sh.weight_before;
                    n_to += sh.n_before;
                    const unsigned long long w_from = w_to - w * num;
                    const uint32_t n_from = n_to - num;
                    if (num && (by_weight ? w_from < target && target <= w_to : n_from < target && target <= n_to)) {
                        const uint32_t j = static_cast<uint32_t>(by_weight ? (target - w_from + w - 1) / w : target - n_from);
                        // zeros of either sign are equal
                        const uint32_t zeros = sh.n[0] + sh.n[kCodes];
                        sh.found_which = place == kCodes ? j + sh.n[0] : j;
                        sh.found_value = value;
                        sh.found_all = value ? num : zeros;
                        sh.found_n = n_from + j;
                        sh.running = w_from + w * j;
                        sh.own = w;
                    }
                }
                __syncthreads();
                found_n = sh.found_n;
                running = sh.running;
            };
            uint32_t kept = all.n;
            unsigned long long total = all.weight;
            narrow(set, kept, total, find);
            if (threadIdx.x < a.parts) {
                const auto tell = [&](uint32_t *p, uint32_t x) { *(a.parts > 1 ? cg::this_cluster().map_shared_rank(p, threadIdx.x) : p) = x; };
                tell(&sh.by_weights, 0u);
                tell(&sh.value, sh.found_value);
                tell(&sh.which, sh.found_all == 1u ? 0u : sh.found_which);
                // of values around zero the first CTA only knows how many there are, not that they are equal
                tell(&sh.around_zero, sh.found_value == 0u);
            }
            if (threadIdx.x == 0) answer(a, r.row, kept, sh.own, total);
        }
    }
    sync();
    if (!sh.by_weights && sh.around_zero) {
        // by their weights if one of them is not zero
        uint32_t tiny = 0;
        r.each_loaded([&](const uint4 &w, uint32_t) {
            const uint32_t *e = reinterpret_cast<const uint32_t *>(&w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t size = (e[i >> 1] >> (16 * (i & 1))) & 0x7fffu;
                tiny |= size != 0u && size <= kFirstCode;
            }
        });
        if (__syncthreads_or(static_cast<int>(tiny)) && threadIdx.x < a.parts) {
            uint32_t *const flag = &sh.tiny;
            *(a.parts > 1 ? cg::this_cluster().map_shared_rank(flag, threadIdx.x) : flag) = 1u;
        }
        sync();
    }
    if (sh.by_weights || sh.tiny) {
        __syncthreads();                                 // the flag has been read: its place is used for other things
        if (a.parts > 1) cg::this_cluster().sync();
        by_weights_rare<R>(a, r.row, part, given_smem);
        return;
    }

    // The column: of `which` (from 1 on; 0: the only one) among those of the value, a run of vectors per warp.
    const uint32_t value = sh.value, which = sh.which;
    const uint32_t bits = value >> 16 | value;           // both halves
    const __nv_bfloat162 wanted = *reinterpret_cast<const __nv_bfloat162 *>(&bits);
    const auto equal = [&](uint32_t w) { return __heq2_mask(*reinterpret_cast<const __nv_bfloat162 *>(&w), wanted); };
    // one bit per element of vector j that has the value
    const auto hits_of = [&](uint4 w, uint32_t j) -> uint32_t {
        uint32_t *const e = reinterpret_cast<uint32_t *>(&w);
        if (!r.whole(j)) {
            w = r.ragged(j);
        } else if constexpr (SCHEME != kSchemeNone) {
            // neither as it is nor with the bias: nothing to hash
            const uint32_t both = a.bias.delta_bf16 | a.bias.delta_bf16 << 16;
            uint32_t near = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) near |= equal(e[i]) | equal(add_bf16x2(e[i], both));
            if (!near) return 0u;
            bias_vector<SBW_DTYPE_BF16, SCHEME>(w, r.rs, a.vocab_offset + r.col0 + j * R::VEC, a.bias);
        }
        uint32_t hits = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t m = equal(e[i]);
            hits |= (m & 1u) << (2 * i) | (m >> 31) << (2 * i + 1);
        }
        return hits;
    };
    constexpr uint32_t kAtOnce = SCHEME == kSchemeNone ? 8 : 4;
    const uint32_t run = (r.vectors + 32 * kGivenWarps - 1) / (32 * kGivenWarps) * 32;      // of a warp, whole trips
    const uint32_t begin = min(warp * run, r.vectors), end = min(begin + run, r.vectors);
    uint32_t mine = 0;
    for (uint32_t j0 = begin + lane; j0 < end; j0 += 32 * kAtOnce) {
        uint4 w[kAtOnce];
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u) {
            const uint32_t j = j0 + 32 * u;
            w[u] = j < end && r.whole(j) ? r.raw(j) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u) {
            const uint32_t j = j0 + 32 * u;
            if (j >= end) break;
            const uint32_t hits = hits_of(w[u], j);
            if (!hits) continue;
            mine += __popc(hits);
            if (which == 0u) put_token(a, r.row, r.col0 + j * R::VEC + __ffs(hits) - 1);
        }
    }
    if (which == 0u) return;
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (lane == 0) sh.warp_ties[warp] = mine;
    __syncthreads();
    uint32_t before = 0, total = 0;
    for (int i = 0; i < kGivenWarps; ++i) {
        if (i < warp) before += sh.warp_ties[i];
        total += sh.warp_ties[i];
    }
    if (a.parts > 1) {
        if (threadIdx.x < a.parts) cg::this_cluster().map_shared_rank(sh.part_ties, threadIdx.x)[part] = total;
        cg::this_cluster().sync();
        for (uint32_t q = 0; q < part; ++q) before += sh.part_ties[q];
    }
    if (which <= before || which > before + mine) return;
    uint32_t left = which - before;                      // from 1 on, among the warp's
    for (uint32_t j0 = begin; j0 < end; j0 += 32) {
        const uint32_t j = j0 + lane;
        const uint32_t hits = j < end ? hits_of(r.whole(j) ? r.raw(j) : make_uint4(0u, 0u, 0u, 0u), j) : 0u;
        const uint32_t own = __popc(hits);
        uint32_t to = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t up = __shfl_up_sync(0xffffffffu, to, d);
            if (lane >= d) to += up;
        }
        const uint32_t all = __shfl_sync(0xffffffffu, to, 31);
        if (left > all) {
            left -= all;
            continue;
        }
        if (to - own < left && left <= to)
            put_token(a, r.row, r.col0 + j * R::VEC + __fns(hits, 0, static_cast<int>(left - (to - own))));
        break;
    }
}

// ---- host -----------------------------------------------------------------------------------

// A launch of clusters of `parts` CTAs.
template <typename K>
struct RowClusters {
    K kernel;
    size_t bytes;              // of shared memory per CTA
    cudaLaunchAttribute attr[1];
    cudaLaunchConfig_t config(int64_t rows, int64_t parts, cudaStream_t stream) {
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = static_cast<unsigned>(parts);
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(static_cast<unsigned>(rows * parts));
        cfg.blockDim = dim3(kGivenThreads);
        cfg.dynamicSmemBytes = bytes;
        cfg.stream = stream;
        cfg.attrs = attr;
        cfg.numAttrs = parts > 1 ? 1 : 0;
        return cfg;
    }
    int launch(const GivenArgs &a, int64_t B, cudaStream_t stream) {
        if (B > 0x7fffffffLL / a.parts) return SBW_ERR_UNSUPPORTED;
        const cudaLaunchConfig_t cfg = config(B, a.parts, stream);
        SBW_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a));
        return SBW_OK;
    }
};

// CTAs per row where any number will do: the most, up to 8, with which all rows are under way at once -- a second round
// costs a row's fixed phases again (37 x 128256 bf16 watermarked: 72 us with 4 CTAs in two rounds, 53 in one with 2) -- as
// long as each finds a vector per thread.  Clusters lie within a GPC, so how many fit is asked, once per device.
template <typename K>
int parts_in_one_round(RowClusters<K> &rows, int64_t B, int64_t row_vectors, int device, std::atomic<int> (&fit)[64][4], int64_t *parts) {
    *parts = 1;
    for (int i = 3; i > 0; --i) {
        const int64_t p = int64_t(1) << i;
        if (row_vectors <= p / 2 * kGivenThreads) continue;
        int n = fit[device][i].load(std::memory_order_acquire);
        if (n == 0) {
            const cudaLaunchConfig_t cfg = rows.config(64, p, nullptr);
            SBW_CUDA_TRY(cudaOccupancyMaxActiveClusters(&n, rows.kernel, &cfg));
            if (n < 1) n = -1;
            fit[device][i].store(n, std::memory_order_release);
        }
        if (B <= n) {
            *parts = p;
            break;
        }
    }
    return SBW_OK;
}

template <int DTYPE, int SCHEME>
int launch_given(GivenArgs &a, int64_t B, cudaStream_t stream) {
    DeviceInfo di;
    if (int rc = current_device_info(&di)) return rc;
    if (di.device >= 64) return SBW_ERR_UNSUPPORTED;
    static std::atomic<uint64_t> prepared{0};
    static std::atomic<int> fit[64][4];
    constexpr int VEC = DTYPE == SBW_DTYPE_F32 ? 4 : 8;
    constexpr bool kByValue = DTYPE == SBW_DTYPE_BF16, kResident = !kByValue && SCHEME != kSchemeNone;
    using Shared = typename Row<DTYPE, SCHEME, kResident>::Shared;
    constexpr size_t kWeights = (sizeof(Shared) + 15) / 16 * 16;
    constexpr size_t kShared = kByValue && sizeof(CodesShared) > kWeights ? sizeof(CodesShared) : kWeights;
    // the most that V, up to its limit, asks of a CTA
    constexpr int64_t kLargest = (kMaxGivenV + 2 * VEC) / VEC * 16 / kMaxParts + 16;
    constexpr int64_t kSlice = !kResident ? 0 : kLargest > kSliceBytes + 16 ? kLargest : kSliceBytes + 16;
    const int64_t row_vectors = (a.V + 2 * (VEC - 1)) / VEC;
    const auto kernel = [] {
        if constexpr (kByValue) return given_codes_kernel<SCHEME>;
        else return given_kernel<DTYPE, SCHEME>;
    }();
    if (!(prepared.load(std::memory_order_acquire) >> di.device & 1)) {
        SBW_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kShared + kSlice)));
        prepared.fetch_or(uint64_t(1) << di.device, std::memory_order_release);
    }
    RowClusters<decltype(kernel)> rows = {kernel, kShared + kSlice, {}};
    int64_t parts;
    if (int rc = parts_in_one_round(rows, B, row_vectors, di.device, fit, &parts)) return rc;
    if (kResident)
        while (parts < kMaxParts && row_vectors * 16 > parts * kSliceBytes) parts *= 2;
    a.parts = static_cast<uint32_t>(parts);
    a.part_vectors = static_cast<uint32_t>((row_vectors + parts - 1) / parts);
    rows.bytes = kShared + (kResident ? static_cast<size_t>(a.part_vectors) * 16 : 0);
    return rows.launch(a, B, stream);
}

}  // namespace
}  // namespace sbw

extern "C" int sbw_sample_given(const void *logits, int dtype, int64_t B, int64_t V, int64_t ld, int64_t vocab_offset,
                                const int32_t *ctx_tokens, int ctx_width, uint64_t key, double gamma, float delta,
                                int scheme, const float *uniforms, const float *temperature, const int32_t *top_k,
                                const float *top_p, const float *min_p, int32_t *out_tokens, float *out_prob,
                                int32_t *out_kept, void *stream) {
    using namespace sbw;
    if (!valid_common(dtype, ctx_width, gamma, scheme)) return SBW_ERR_INVALID_ARG;
    if (B < 0 || V <= 0 || ld < V || vocab_offset < 0) return SBW_ERR_INVALID_ARG;
    if (!(delta == delta) || delta - delta != 0.0f) return SBW_ERR_INVALID_ARG;
    if (vocab_offset + V > (int64_t(1) << 32)) return SBW_ERR_UNSUPPORTED;
    if (V > kMaxGivenV) return SBW_ERR_TOO_LARGE;
    if (B == 0) return SBW_OK;
    const float in_precision = dtype == SBW_DTYPE_BF16 ? __bfloat162float(__float2bfloat16_rn(delta)) : delta;
    const bool marked = in_precision != 0.0f;
    if (!logits || !uniforms || !temperature || !out_tokens || (marked && !ctx_tokens)) return SBW_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(logits) % (dtype == SBW_DTYPE_F32 ? 4 : 2) != 0) return SBW_ERR_INVALID_ARG;
    GivenArgs a = {};
    a.logits = logits;
    a.B = B;
    a.V = V;
    a.ld = ld;
    a.vocab_offset = static_cast<uint32_t>(vocab_offset);
    a.ctx = ctx_tokens;
    a.W = ctx_width;
    a.bias.key = key;
    a.bias.thr_m1 = threshold_minus_one(gamma);
    a.bias.delta = in_precision;
    a.bias.delta_bf16 = dtype == SBW_DTYPE_BF16 ? static_cast<uint32_t>(__bfloat16_as_ushort(__float2bfloat16_rn(delta))) : 0u;
    a.bias.weyl = make_weyl();
    a.uniforms = uniforms;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.out_tokens = out_tokens;
    a.out_prob = out_prob;
    a.out_kept = out_kept;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == SBW_DTYPE_F32) {
        if (!marked) return launch_given<SBW_DTYPE_F32, kSchemeNone>(a, B, s);
        return scheme == SBW_SCHEME_CONTEXT ? launch_given<SBW_DTYPE_F32, SBW_SCHEME_CONTEXT>(a, B, s)
                                            : launch_given<SBW_DTYPE_F32, SBW_SCHEME_SELFSALT>(a, B, s);
    }
    if (!marked) return launch_given<SBW_DTYPE_BF16, kSchemeNone>(a, B, s);
    return scheme == SBW_SCHEME_CONTEXT ? launch_given<SBW_DTYPE_BF16, SBW_SCHEME_CONTEXT>(a, B, s)
                                        : launch_given<SBW_DTYPE_BF16, SBW_SCHEME_SELFSALT>(a, B, s);
}
