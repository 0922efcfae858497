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
// A row is read from memory once.  A cluster of CTAs keeps its biased logits in shared memory, a slice
// per CTA, and passes over them there:
//   maximum    while loading
//   histogram  1024 bins by the weight's exponent and six bits of its mantissa, down to 2^-16 of the
//              maximum: the number of candidates and the sum of the other 17 bits (32-bit counters, native
//              adds).  Weights below that are summed in registers.
//   lists      the first CTA scans the bins, asks the others for the candidates of the first bins up to
//              the one that is looked for (of that bin alone if those are too many for the list), sorts
//              them and walks the running sums.  The first list usually answers all questions.
// A bin too full for the list is split by the candidates' bits, 1024 ways at a time; candidates of equal
// value, however many, are counted by column.
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
constexpr int64_t kSliceBytes = 68 * 1024;           // two CTAs with such a slice fit on an SM
// A sum of 17 bits holds 32768 candidates: every other warp of a CTA has its own.  The tail's sums in
// registers hold 128 weights of 25 bits.
static_assert(kMaxGivenV / kMaxParts <= 61440 && kSliceBytes / 2 <= 61440, "");
static_assert(kMaxGivenV / kMaxParts + 16 <= 120 * kGivenThreads && kSliceBytes / 2 <= 120 * kGivenThreads, "");
constexpr uint32_t kLimb = 12;                       // of a split's two sums

struct GivenArgs {
    const void *logits;
    int64_t V, ld;
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
struct GivenShared {
    struct {
        uint32_t n[kBins], low[2][kBins];
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
__device__ __forceinline__ void power(Pair y, uint32_t &v0, uint32_t &v1) {
    const Pair t = pair_add(y, pair_of(kRound, kRound));
    const Pair f = pair_fma(pair_add(t, pair_of(-kRound, -kRound)), pair_of(-1.0f, -1.0f), y);
    Pair p = pair_of(0x1.ffcbfcp+23f, 0x1.ffcbfcp+23f);
    p = pair_fma(p, f, pair_of(0x1.430912p+27f, 0x1.430912p+27f));
    p = pair_fma(p, f, pair_of(0x1.5d87fep+30f, 0x1.5d87fep+30f));
    p = pair_fma(p, f, pair_of(0x1.3b2ab6p+33f, 0x1.3b2ab6p+33f));
    p = pair_fma(p, f, pair_of(0x1.c6b08ep+35f, 0x1.c6b08ep+35f));
    p = pair_fma(p, f, pair_of(0x1.ebfbep+37f, 0x1.ebfbep+37f));
    p = pair_fma(p, f, pair_of(0x1.62e43p+39f, 0x1.62e43p+39f));
    p = pair_fma(p, f, pair_of(0x1p+40f, 0x1p+40f));
    float p0, p1, t0, t1;
    of_pair(p, p0, p1);
    of_pair(t, t0, t1);
    v0 = __float_as_uint(p0) + (__float_as_uint(t0) << 23);      // the low bits of kRound are 0: n goes to the exponent
    v1 = __float_as_uint(p1) + (__float_as_uint(t1) << 23);
}
__device__ __forceinline__ uint32_t power(float y) {
    uint32_t v, other;
    power(pair_of(y, y), v, other);
    return v;
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

template <int DTYPE>
struct Row {
    static constexpr int VEC = DTYPE == SBW_DTYPE_F32 ? 4 : 8;
    const uint4 *slice;        // this CTA's vectors
    uint32_t vectors;
    uint32_t col0;             // column of its first element; columns before 0 wrap, their values are -inf
    static __device__ __forceinline__ float value(const uint4 &w, int i) {
        const uint32_t *e = reinterpret_cast<const uint32_t *>(&w);
        if constexpr (DTYPE == SBW_DTYPE_F32) return __uint_as_float(e[i]);
        else return __uint_as_float((i & 1) ? (e[i >> 1] & 0xffff0000u) : (e[i >> 1] << 16));
    }
    // Element i of the thread's vector w, and the next, as a pair.
    static __device__ __forceinline__ Pair values(const uint4 &w, int i) { return pair_of(value(w, i), value(w, i + 1)); }
};

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

// Loads this CTA's slice of the row, biased, and returns the thread's largest value.
template <int DTYPE, int SCHEME>
__device__ __forceinline__ float load_slice(const GivenArgs &a, int64_t row, uint4 *slice, uint32_t vec0, uint32_t vectors, uint32_t head) {
    constexpr int VEC = Row<DTYPE>::VEC;
    constexpr int kInFlight = SCHEME == kSchemeNone ? 8 : 2;
    const char *const row_ptr = static_cast<const char *>(a.logits) + row * a.ld * (16 / VEC);
    const char *const base = row_ptr - static_cast<int64_t>(head) * (16 / VEC);     // 16-byte aligned
    RowSeedS<SCHEME> rs;
    rs.init(a.bias.key, a.ctx + row * a.W, a.W);
    const uint32_t V = static_cast<uint32_t>(a.V);
    float best = -INFINITY;
    for (uint32_t j0 = threadIdx.x; j0 < vectors; j0 += kInFlight * kGivenThreads) {
        uint4 w[kInFlight];
        bool whole[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const uint32_t j = j0 + u * kGivenThreads, first = (vec0 + j) * VEC;      // of its elements, head included
            whole[u] = j < vectors && first >= head && first + VEC <= head + V;
            w[u] = whole[u] ? __ldcs(reinterpret_cast<const uint4 *>(base) + vec0 + j) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const uint32_t j = j0 + u * kGivenThreads;
            if (j >= vectors) break;
            const uint32_t col = (vec0 + j) * VEC - head;
            if (whole[u]) {
                bias_vector<DTYPE, SCHEME>(w[u], rs, a.vocab_offset + col, a.bias);
            } else {
                uint32_t *e = reinterpret_cast<uint32_t *>(&w[u]);
#pragma unroll 1
                for (int i = 0; i < VEC; ++i) {
                    float x = -INFINITY;
                    if (col + i < V) x = biased_at<DTYPE, SCHEME>(row_ptr, col + i, rs, a.vocab_offset + col + i, a.bias);
                    if constexpr (DTYPE == SBW_DTYPE_F32) e[i] = __float_as_uint(x);
                    else e[i >> 1] |= (i & 1) ? (__float_as_uint(x) & 0xffff0000u) : (__float_as_uint(x) >> 16);
                }
            }
            settle<DTYPE>(w[u]);
            slice[j] = w[u];
#pragma unroll
            for (int i = 0; i < VEC; ++i) best = fmaxf(best, Row<DTYPE>::value(w[u], i));
        }
    }
    return best;
}

// One add to shared memory under a condition, as a predicated instruction: a branch per element would keep the
// elements of a vector from overlapping.
__device__ __forceinline__ void add_if(bool yes, uint32_t addr, uint32_t x) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p red.relaxed.cta.shared::cta.add.u32 [%0], %1;\n\t}"
                 ::"r"(addr), "r"(x), "r"(static_cast<uint32_t>(yes)) : "memory");
}

template <int DTYPE>
class Cluster {
  public:
    GivenShared &sh;
    const Row<DTYPE> row;
    const RowWeights rw;
    const uint32_t parts, part;

    __device__ __forceinline__ Cluster(GivenShared &s, const Row<DTYPE> &r, const RowWeights &w, uint32_t n, uint32_t p)
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
        for (int i = threadIdx.x; i < kBins; i += kGivenThreads) sh.hist.n[i] = sh.hist.low[0][i] = sh.hist.low[1][i] = 0u;
        __syncthreads();
        // addresses less what the first bin's bits come to
        const uint32_t at_n = static_cast<uint32_t>(__cvta_generic_to_shared(sh.hist.n)) - 4u * kFirstBits;
        const uint32_t at_low = static_cast<uint32_t>(__cvta_generic_to_shared(sh.hist.low[(threadIdx.x >> 5) & 1])) - 4u * kFirstBits;
        uint32_t tail = 0, number = 0;
        for (uint32_t j = threadIdx.x; j < row.vectors; j += kGivenThreads) {
            const uint4 w = row.slice[j];
#pragma unroll
            for (int i = 0; i < Row<DTYPE>::VEC; i += 2) {
                const Pair y = log2_of(Row<DTYPE>::values(w, i));
                float yy[2];
                uint32_t v[2];
                of_pair(y, yy[0], yy[1]);
                power(y, v[0], v[1]);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t u = yy[k] >= rw.lowest ? v[k] : 0u;
                    const bool binned = u >= kFirstBits << kLowBits;
                    const uint32_t four_bin = u >> (kLowBits - 2) & ~3u;
                    add_if(binned, at_n + four_bin, 1u);
                    add_if(binned, at_low + four_bin, u & ((1u << kLowBits) - 1u));
                    const uint32_t whole = binned ? 0u : __float2uint_rz(__uint_as_float(u));
                    tail += whole;
                    number += whole != 0u;
                }
            }
        }
        // n and weight of the tail to the first CTA
        Sums total;
        block_before(tail, number, sh.scan, total);
        if (threadIdx.x == 0) {
            at(sh.tail_weight, 0)[part] = total.weight;
            at(sh.tail_n, 0)[part] = total.n;
        }
    }

    // Every CTA adds up a share of the bins over all CTAs and hands it to the first.
    __device__ __forceinline__ void merge() const {
        sync();
        const uint32_t share = kBins / parts;            // a power of two
        for (uint32_t i = threadIdx.x; i < share; i += kGivenThreads) {
            const uint32_t bin = part * share + i;
            uint32_t n = 0;
            unsigned long long low = 0;
#pragma unroll
            for (uint32_t r = 0; r < kMaxParts; ++r) {       // unrolled: the loads from other SMs overlap
                if (r >= parts) break;
                n += *at(&sh.hist.n[bin], r);
                low += static_cast<unsigned long long>(*at(&sh.hist.low[0][bin], r)) + *at(&sh.hist.low[1][bin], r);
            }
            const uint32_t v = (bin + kFirstBits) << kLowBits;       // the bin's least weight
            *at(&sh.bins.n[bin], 0) = n;
            *at(&sh.bins.weight[bin], 0) =
                (static_cast<unsigned long long>(n) * ((v & 0x7fffffu) | 0x800000u) + low) << shift_of_bin(static_cast<int>(bin));
        }
        sync();
    }

    // f(value, column, weight's bits, distance) for the candidates that a command names.
    template <typename F>
    __device__ __forceinline__ void each_named(const Command &c, F f) const {
        constexpr int VEC = Row<DTYPE>::VEC;
        // log2 of the bins' ends, with a margin for the rounding of y and of the logarithm
        const float from = c.bin_lo == kTail ? rw.lowest
                                             : fmaxf(rw.lowest, __log2f(__uint_as_float((c.bin_lo + kFirstBits) << kLowBits)) - 40.01f);
        const float to = __log2f(__uint_as_float((c.bin_hi + 1 + kFirstBits) << kLowBits)) - 39.99f;
        for (uint32_t j = threadIdx.x; j < row.vectors; j += kGivenThreads) {
            const uint4 w = row.slice[j];
            uint32_t hits = 0;
#pragma unroll
            for (int i = 0; i < VEC; i += 2) {
                float y0, y1;
                of_pair(log2_of(Row<DTYPE>::values(w, i)), y0, y1);
                if (y0 >= from && y0 <= to) hits |= 1u << i;
                if (y1 >= from && y1 <= to) hits |= 2u << i;
            }
            while (hits) {
                const int i = __ffs(hits) - 1;
                hits &= hits - 1u;
                const float x = Row<DTYPE>::value(row.slice[j], i);
                const uint32_t v = power(rw.log2_of(x)), dist = distance(x);
                const int bin = bin_of(v);
                if (bin >= c.bin_lo && bin <= c.bin_hi && dist >= c.dist_lo && dist <= c.dist_hi) f(row.col0 + j * VEC + i, v, dist);
            }
        }
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
                    if (first + i < kListCap) list[first + i] = sh.list[i];
            }
        } else if (c.op == kSplit) {
            if (part != 0) {                             // the first CTA has cleared its own
                for (int i = threadIdx.x; i < kFine; i += kGivenThreads) sh.fine.n[i] = sh.fine.lo[i] = sh.fine.hi[i] = 0u;
                __syncthreads();
            }
            each_named(c, [&](uint32_t, uint32_t v, uint32_t dist) {
                const uint32_t bin = (dist - c.dist_lo) >> c.shift;
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
            constexpr int VEC = Row<DTYPE>::VEC;
            const float x = __uint_as_float(order_decode(rw.code_m - c.dist_lo));
            const uint32_t run = (row.vectors + kGivenThreads - 1) / kGivenThreads;
            const uint32_t begin = min(threadIdx.x * run, row.vectors), end = min(begin + run, row.vectors);
            uint32_t mine = 0;
            for (uint32_t j = begin; j < end; ++j) {
                const uint4 w = row.slice[j];
#pragma unroll
                for (int i = 0; i < VEC; ++i) mine += Row<DTYPE>::value(w, i) == x;
            }
            Sums total;
            const uint32_t before = block_before(0ull, mine, sh.scan, total).n;
            if (c.op == kCountTies) {
                if (threadIdx.x == 0) at(sh.ties, 0)[part] = total.n;
            } else if (c.part == part && before <= c.which && c.which < before + mine) {
                uint32_t left = c.which - before;
                for (uint32_t j = begin; j < end; ++j) {
                    const uint4 w = row.slice[j];
#pragma unroll 1
                    for (int i = 0; i < VEC; ++i)
                        if (Row<DTYPE>::value(w, i) == x && left-- == 0u) *at(&sh.tie_col, 0) = row.col0 + j * VEC + i;
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
template <int DTYPE>
class Finder {
    static constexpr int kOwn = kBins / kGivenThreads, kOwnFine = kFine / kGivenThreads, kOwnList = kListCap / kGivenThreads;
    const Cluster<DTYPE> &cl;
    GivenShared &sh;
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

    __device__ __forceinline__ explicit Finder(const Cluster<DTYPE> &c) : cl(c), sh(c.sh) {
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
    __device__ __noinline__ Found find(bool by_weight, unsigned long long target) {
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
            if (threadIdx.x < list_n) sh.list[rank] = mine;
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

template <int DTYPE, int SCHEME>
__global__ void __launch_bounds__(kGivenThreads, SCHEME == kSchemeNone ? 2 : 1) given_kernel(const GivenArgs a) {
    constexpr int VEC = Row<DTYPE>::VEC;
    extern __shared__ __align__(16) uint8_t given_smem[];
    __shared__ GivenShared sh;
    uint4 *const slice = reinterpret_cast<uint4 *>(given_smem);
    const int64_t row = blockIdx.x / a.parts;
    const uint32_t part = blockIdx.x % a.parts;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (a.parts > 1) cg::this_cluster().barrier_arrive();

    // the row's vectors start at the 16-byte boundary at or before it
    const uintptr_t row_at = reinterpret_cast<uintptr_t>(a.logits) + static_cast<uintptr_t>(row * a.ld) * (16 / VEC);
    const uint32_t head = static_cast<uint32_t>(row_at % 16) / (16 / VEC);
    const uint32_t row_vectors = (head + static_cast<uint32_t>(a.V) + VEC - 1) / VEC;
    const uint32_t vec0 = min(part * a.part_vectors, row_vectors);
    const uint32_t vectors = min(a.part_vectors, row_vectors - vec0);

    float m = load_slice<DTYPE, SCHEME>(a, row, slice, vec0, vectors, head);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    if (lane == 0) sh.warp_max[warp] = m;
    __syncthreads();
    if (a.parts > 1) {
        cg::this_cluster().barrier_wait();               // every CTA has begun: its shared memory can be written
        if (threadIdx.x < a.parts) {
            for (int w = 1; w < kGivenWarps; ++w) m = fmaxf(m, sh.warp_max[w]);
            m = fmaxf(m, sh.warp_max[0]);
            cg::this_cluster().map_shared_rank(sh.part_max, threadIdx.x)[part] = m;
        }
        cg::this_cluster().sync();
        m = sh.part_max[0];
        for (uint32_t r = 1; r < a.parts; ++r) m = fmaxf(m, sh.part_max[r]);
    } else {
        for (int w = 0; w < kGivenWarps; ++w) m = fmaxf(m, sh.warp_max[w]);
    }
    if (m == -INFINITY) {                                // nothing can be drawn: every CTA of the cluster sees it
        if (part == 0 && threadIdx.x == 0) {
            a.out_tokens[row] = 0;
            if (a.out_prob) a.out_prob[row] = 0.0f;
            if (a.out_kept) a.out_kept[row] = 0;
        }
        return;
    }
    if (m == INFINITY) {                                 // the infinite ones share everything
        for (uint32_t j = threadIdx.x; j < vectors; j += kGivenThreads) {
            uint32_t *e = reinterpret_cast<uint32_t *>(&slice[j]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (DTYPE == SBW_DTYPE_F32) {
                    e[i] = e[i] == 0x7f800000u ? 0u : 0xff800000u;
                } else {
                    e[i] = ((e[i] & 0xffffu) == 0x7f80u ? 0u : 0xff80u) | ((e[i] >> 16) == 0x7f80u ? 0u : 0xff800000u);
                }
            }
        }
        __syncthreads();
        m = 0.0f;
    }

    // the row's settings
    const float tau = a.temperature[row];
    const bool greedy = !(tau >= 1e-6f);
    RowWeights rw;
    rw.m = m;
    rw.code_m = order_code(__float_as_uint(m));
    rw.c = greedy ? 1.0f : static_cast<float>(1.4426950408889634 / static_cast<double>(tau));
    rw.lowest = -40.0f;                                  // below that a weight is 0
    if (!greedy && a.min_p && a.min_p[row] > 0.0f)
        rw.lowest = fminf(fmaxf(static_cast<float>(log2(static_cast<double>(a.min_p[row]))), -40.0f), 0.0f);

    Row<DTYPE> r;
    r.slice = slice;
    r.vectors = vectors;
    r.col0 = vec0 * VEC - head;
    const Cluster<DTYPE> cl(sh, r, rw, a.parts, part);
    cl.histogram();
    cl.merge();
    if (part != 0) {
        cl.serve();
        return;
    }
    Finder<DTYPE> finder(cl);
    const int64_t k = greedy ? 1 : a.top_k ? a.top_k[row] : 0;
    uint32_t kept = finder.total_n;
    unsigned long long total = finder.total_w;
    if (k > 0 && k < kept) {
        const Found f = finder.find(false, static_cast<unsigned long long>(k));
        kept = f.n;
        total = f.running;
    }
    if (!greedy && a.top_p && a.top_p[row] < 1.0f) {
        const double p = floor(static_cast<double>(a.top_p[row]) * 4294967296.0);
        bool rest;
        unsigned long long need = share_of(p >= 1.0 ? static_cast<unsigned long long>(p) : 1ull, total, rest);
        need += rest;
        if (need < total) {
            const Found f = finder.find(true, need);
            kept = f.n;
            total = f.running;
        }
    }
    const double u = static_cast<double>(a.uniforms[row]) * 4294967296.0;
    const unsigned long long u32 = u >= 4294967295.0 ? 0xffffffffull : u >= 1.0 ? static_cast<unsigned long long>(u) : 0ull;
    bool rest;
    const Found f = finder.find(true, share_of(u32, total, rest) + 1ull);
    if (threadIdx.x == 0) {
        a.out_tokens[row] = static_cast<int32_t>(f.col);
        if (a.out_prob) a.out_prob[row] = static_cast<float>(static_cast<double>(f.own) / static_cast<double>(total));
        if (a.out_kept) a.out_kept[row] = static_cast<int32_t>(kept);
    }
    Command done = {};
    cl.order(done);
}

// ---- host -----------------------------------------------------------------------------------

template <int DTYPE, int SCHEME>
int launch_given(GivenArgs &a, int64_t B, cudaStream_t stream) {
    constexpr int VEC = Row<DTYPE>::VEC;
    DeviceInfo di;
    if (int rc = current_device_info(&di)) return rc;
    // CTAs per row: so many that two of them fit on an SM (one row's passes over shared memory then run
    // beside another row's loads), and more where few rows would leave SMs without work
    const int64_t row_vectors = (a.V + 2 * (VEC - 1)) / VEC;
    int64_t parts = 1;
    while (parts < kMaxParts && (row_vectors * 16 > parts * kSliceBytes || (B * parts * 2 <= di.sm_count && row_vectors > parts * kGivenThreads)))
        parts *= 2;
    a.parts = static_cast<uint32_t>(parts);
    a.part_vectors = static_cast<uint32_t>((row_vectors + parts - 1) / parts);
    if (B > 0x7fffffffLL / parts) return SBW_ERR_UNSUPPORTED;
    const size_t bytes = static_cast<size_t>(a.part_vectors) * 16;
    const auto kernel = given_kernel<DTYPE, SCHEME>;
    static std::atomic<uint64_t> prepared{0};
    if (!(prepared.load(std::memory_order_acquire) >> di.device & 1)) {
        // the most that V, up to its limit, asks of a CTA
        constexpr int64_t kLargest = (kMaxGivenV + 2 * VEC) / VEC * 16 / kMaxParts + 16;
        constexpr int kMost = static_cast<int>(kLargest > kSliceBytes + 16 ? kLargest : kSliceBytes + 16);
        SBW_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost));
        prepared.fetch_or(uint64_t(1) << di.device, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(B * parts));
    cfg.blockDim = dim3(kGivenThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(parts);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = parts > 1 ? 1 : 0;
    SBW_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, a));
    return SBW_OK;
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
