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
#include <cooperative_groups.h>

#include <cfloat>
#include <cmath>

#include "sbw_codes.cuh"
#include "sbw_common.cuh"
#include "sbw_rowbias.cuh"

namespace sbw {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kGroups = kThreads / 4;   // maxima of disjoint column sets that bound the alternatives from below
constexpr int kCap = 2048;              // candidate list entries
constexpr int kMaxTop = SBW_MAX_TOP_LOGPROBS;
constexpr int kMaxCluster = 8;
constexpr float kFar = -300.0f;         // exponents below this give 2^x = 0; keeps 0 * inf out of the sums
static_assert(kCap >= 32 * kMaxTop, "a row with fewer groups than alternatives must fit the list");

struct LogprobArgs {
    const void *logits;
    int64_t B, V, ld;
    const int32_t *ctx;
    int W;
    uint32_t vocab_offset;
    BiasParams bias;
    double tau;
    float c;               // log2(e) / tau
    const int32_t *tokens; // nullable
    int top_n;
    float *out_logprob, *out_entropy;
    int32_t *out_rank;
    float *out_max, *out_sumexp;
    int32_t *out_top_ids;
    float *out_top_logprobs;
};

// ---- two fp32 operations per instruction ----
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t p, float &lo, float &hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p));
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
// max that keeps a NaN (fmaxf drops it): a NaN logit has to reach the sums
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
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

struct Stats {
    float m, z, s;    // reference (a maximum, at least -FLT_MAX), sum, first moment in log2 units
    uint32_t above;   // columns that rank before the token
    // the same sums with reference `to` >= m
    __device__ __forceinline__ void move(float to, float c) {
        const float d = fmaxf((m - to) * c, kFar);
        const float f = ex2_approx_ftz(d);
        s = f * fmaf(d, z, s);
        z *= f;
        m = to;
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

template <int DTYPE>
__device__ __forceinline__ float element(const uint4 &w, int i) {
    const uint32_t *e = reinterpret_cast<const uint32_t *>(&w);
    if constexpr (DTYPE == SBW_DTYPE_F32) return __uint_as_float(e[i]);
    else return __uint_as_float((i & 1) ? e[i >> 1] & 0xffff0000u : e[i >> 1] << 16);
}

__device__ __forceinline__ uint4 load_vector(const uint4 *p) {
    uint4 r;   // read once: no need to keep it in L1
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

__device__ __forceinline__ uint4 load_vector_rw(const uint4 *p) {
    uint4 r;   // the same where the kernel may write over what it has read
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
    return r;
}

// ---- the seldom taken passes over the columns [lo, hi) of a row: plain, one column at a time, out of
// line so that the common path's registers do not pay for them ----
template <int DTYPE, int SCHEME>
struct Columns {
    const LogprobArgs &a;
    const char *row_ptr;
    RowSeedS<SCHEME> rs;
    __device__ __forceinline__ Columns(const LogprobArgs &args, int64_t row)
        : a(args), row_ptr(static_cast<const char *>(args.logits) + row * args.ld * RowLayout<DTYPE>::ESIZE) {
        rs.init(args.bias.key, args.ctx + row * args.W, args.W);
    }
    __device__ __forceinline__ float operator[](uint32_t col) const {
        return biased_at<DTYPE, SCHEME>(row_ptr, col, rs, a.vocab_offset + col, a.bias);
    }
};

// Columns that rank before column t when its value is -inf (or NaN, which counts as that).
template <int DTYPE, int SCHEME>
__device__ __noinline__ uint32_t count_above_nothing(const LogprobArgs &a, int64_t row, uint32_t lo, uint32_t hi, uint32_t t) {
    const Columns<DTYPE, SCHEME> x(a, row);
    uint32_t n = 0;
    for (uint32_t col = lo + threadIdx.x; col < hi; col += kThreads) n += (x[col] > -INFINITY || col < t) ? 1u : 0u;
    return n;
}

// Candidates strictly above `floor`.
template <int DTYPE, int SCHEME>
__device__ __noinline__ void gather_above(const LogprobArgs &a, int64_t row, uint32_t lo, uint32_t hi, float floor, uint64_t *list,
                                          unsigned *count) {
    const Columns<DTYPE, SCHEME> x(a, row);
    for (uint32_t col = lo + threadIdx.x; col < hi; col += kThreads) {
        const float v = x[col];
        if (v > floor) {
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
        for (uint32_t col = lo + threadIdx.x; col < hi; col += kThreads) {
            const uint64_t e = composite(x[col], col);
            if (e < last && e > best) best = e;
        }
        for (int d = 16; d > 0; d >>= 1) {
            const uint64_t o = __shfl_xor_sync(0xffffffffu, best, d);
            best = o > best ? o : best;
        }
        if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = best;
        __syncthreads();
        for (int w = 0; w < kWarps; ++w) best = scratch[w] > best ? scratch[w] : best;
        if (threadIdx.x == 0) list[r] = best;
        last = best;
        __syncthreads();
    }
}

// One CTA per row for large batches, a cluster of up to 8 CTAs per row for small ones: each CTA
// takes a share of the row's vectors, and CTA 0 merges the others' sums and alternatives out of
// their shared memory.  No workspace, no atomics outside a CTA, one launch.
template <int DTYPE, int SCHEME, bool TOP>
__global__ void __launch_bounds__(kThreads, SCHEME == kSchemeNone ? 2 : 1)
logprob_kernel(const __grid_constant__ LogprobArgs a) {
    namespace cg = cooperative_groups;
    using Layout = RowLayout<DTYPE>;
    constexpr int VEC = Layout::VEC;
    constexpr int U = SCHEME == kSchemeNone ? 4 : 2;    // vectors in flight per thread
    __shared__ Stats sh_warp[kWarps];
    __shared__ Stats sh_part;
    __shared__ float sh_group[TOP ? kGroups : 1];
    __shared__ float sh_floor;
    __shared__ unsigned sh_count;
    __shared__ uint64_t sh_scratch[kWarps];
    __shared__ uint64_t sh_list[TOP ? kCap : 1];
    __shared__ uint64_t sh_top[TOP ? kMaxTop : 1];      // this part's alternatives, best first, 0 = none
    __shared__ uint64_t sh_all[TOP ? kMaxTop * kMaxCluster : 1];

    const auto cluster = cg::this_cluster();
    const unsigned parts = cluster.num_blocks(), part = cluster.block_rank();
    const uint32_t V = static_cast<uint32_t>(a.V);
    const float c = a.c;
    const uint64_t c2 = pack2(c, c);
    const unsigned tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    for (int64_t row = blockIdx.x / parts; row < a.B; row += gridDim.x / parts) {
        const char *row_ptr = static_cast<const char *>(a.logits) + row * a.ld * Layout::ESIZE;
        const uint32_t t = a.tokens ? static_cast<uint32_t>(a.tokens[row]) : 0u;
        if (a.tokens && t >= V) {                        // a padded row: every CTA of the cluster skips it
            if (part == 0) {
                if (tid == 0) {
                    if (a.out_logprob) a.out_logprob[row] = 0.0f;
                    if (a.out_entropy) a.out_entropy[row] = 0.0f;
                    if (a.out_rank) a.out_rank[row] = 0;
                    if (a.out_max) a.out_max[row] = 0.0f;
                    if (a.out_sumexp) a.out_sumexp[row] = 0.0f;
                }
                for (unsigned i = tid; TOP && i < static_cast<unsigned>(a.top_n); i += kThreads) {
                    if (a.out_top_ids) a.out_top_ids[row * a.top_n + i] = -1;
                    if (a.out_top_logprobs) a.out_top_logprobs[row * a.top_n + i] = -INFINITY;
                }
            }
            continue;
        }
        RowSeedS<SCHEME> rs;
        rs.init(a.bias.key, a.ctx + row * a.W, a.W);
        const Layout layout(row_ptr, V);
        const uint4 *vectors = reinterpret_cast<const uint4 *>(row_ptr + static_cast<size_t>(layout.head) * Layout::ESIZE);
        const uint32_t v_lo = static_cast<uint32_t>(static_cast<uint64_t>(layout.nvec) * part / parts);
        const uint32_t v_hi = static_cast<uint32_t>(static_cast<uint64_t>(layout.nvec) * (part + 1) / parts);
        // this part's columns: its vectors, and the ragged ends with the first and the last part
        const uint32_t c_lo = part == 0 ? 0u : layout.head + v_lo * VEC;
        const uint32_t c_hi = part + 1 == parts ? V : layout.head + v_hi * VEC;

        // the token's own value, and the values its rank is counted against: strictly greater ones
        // from its column on, before it also equal ones (greater than the next value below)
        const bool ranked = a.tokens != nullptr && a.out_rank != nullptr;
        float xt = INFINITY;
        if (a.tokens) xt = biased_at<DTYPE, SCHEME>(row_ptr, t, rs, a.vocab_offset + t, a.bias);
        const bool t_nothing = ranked && !(xt > -INFINITY);
        const float bar = ranked && !t_nothing ? xt : INFINITY;

        Stats st = {-FLT_MAX, 0.0f, 0.0f, 0u};
        uint64_t z2 = 0, s2 = 0;                         // pairs of partial sums
        float floor = INFINITY;                          // alternatives have at least this value

        auto fold = [&]() {                              // z2, s2 into st
            float lo, hi;
            unpack2(z2, lo, hi);
            st.z += lo + hi;
            unpack2(s2, lo, hi);
            st.s += lo + hi;
            z2 = s2 = 0;
        };
        auto push = [&](float x, uint32_t col) {
            if (x >= floor && x > -INFINITY) {
                const unsigned pos = atomicAdd(&sh_count, 1u);
                if (pos < static_cast<unsigned>(kCap)) sh_list[pos] = composite(x, col);
            }
        };

        // ragged ends: at most one column per thread
        float xe = -INFINITY;
        uint32_t ce = V;
        {
            const uint32_t first_tail = layout.head + layout.nvec * VEC;
            if (part == 0 && tid < layout.head) ce = tid;
            else if (part + 1 == parts && tid >= 32 && tid - 32 < V - first_tail) ce = first_tail + tid - 32;
            if (ce < V) {
                xe = biased_at<DTYPE, SCHEME>(row_ptr, ce, rs, a.vocab_offset + ce, a.bias);
                if (xe > st.m) st.m = xe;
                const float x = max_nan((xe - st.m) * c, kFar);
                const float e = ex2_approx_ftz(x);
                st.z += e;
                st.s = fmaf(e, x, st.s);
                if (xe > bar || (xe == bar && ce < t)) st.above += 1u;
            }
        }

        const uint32_t n_vec = v_hi - v_lo;
        const uint32_t trips = max(1u, (n_vec + U * kThreads - 1) / (U * kThreads));
        for (uint32_t trip = 0; trip < trips; ++trip) {
            const uint32_t j0 = v_lo + trip * (U * kThreads) + tid;
            uint4 w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t j = j0 + u * kThreads;
                const uint32_t none = DTYPE == SBW_DTYPE_F32 ? 0xff800000u : 0xff80ff80u;
                w[u] = j < v_hi ? load_vector(vectors + j) : make_uint4(none, none, none, none);
            }
            float vm[U];
            float mx = -INFINITY;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t col = layout.head + (j0 + u * kThreads) * VEC;
                bias_vector<DTYPE, SCHEME>(w[u], rs, a.vocab_offset + col, a.bias);
                vm[u] = vector_max<DTYPE>(w[u]);
                mx = fmaxf(mx, vm[u]);
            }
            if (mx > st.m) st.move(mx, c);
            const uint64_t nm2 = pack2(-st.m, -st.m);
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int i = 0; i < VEC; i += 2) {
                    float x0, x1;
                    unpack2(mul2(add2(pack2(element<DTYPE>(w[u], i), element<DTYPE>(w[u], i + 1)), nm2), c2), x0, x1);
                    x0 = max_nan(x0, kFar);
                    x1 = max_nan(x1, kFar);
                    const uint64_t e = pack2(ex2_approx_ftz(x0), ex2_approx_ftz(x1));
                    z2 = add2(z2, e);
                    s2 = fma2(e, pack2(x0, x1), s2);
                }
                if (vm[u] >= bar) {
                    const uint32_t col = layout.head + (j0 + u * kThreads) * VEC;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        const float x = element<DTYPE>(w[u], i);
                        if (x > bar || (x == bar && col + i < t)) st.above += 1u;
                    }
                }
            }
            fold();                                      // short chains of additions: a trip's, then the trips'
            if constexpr (TOP) {
                if (trip == 0) {
                    // the top_n-th largest of 128 maxima of disjoint column sets bounds this part's
                    // alternatives from below; known after the first trip
                    float g = fmaxf(mx, xe);
                    g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 1));
                    g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 2));
                    if ((lane & 3) == 0) sh_group[tid >> 2] = g;
                    if (tid == 0) sh_count = 0;
                    __syncthreads();
                    if (tid < static_cast<unsigned>(kGroups)) {
                        const float mine = sh_group[tid];
                        int rank = 0;
                        for (int o = 0; o < kGroups; ++o) {
                            const float other = sh_group[o];
                            rank += (other > mine || (other == mine && o < static_cast<int>(tid))) ? 1 : 0;
                        }
                        if (rank == a.top_n - 1) sh_floor = mine;
                    }
                    __syncthreads();
                    floor = sh_floor;
                    if (ce < V) push(xe, ce);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (vm[u] >= floor && j0 + u * kThreads < v_hi) {
                        const uint32_t col = layout.head + (j0 + u * kThreads) * VEC;
#pragma unroll
                        for (int i = 0; i < VEC; ++i) push(element<DTYPE>(w[u], i), col + i);
                    }
                }
            }
        }
        if (t_nothing) st.above = count_above_nothing<DTYPE, SCHEME>(a, row, c_lo, c_hi, t);

        // ---- this part's sums ----
        {
            float m = st.m;
            for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
            st.move(m, c);
            for (int d = 16; d > 0; d >>= 1) {
                st.z += __shfl_xor_sync(0xffffffffu, st.z, d);
                st.s += __shfl_xor_sync(0xffffffffu, st.s, d);
                st.above += __shfl_xor_sync(0xffffffffu, st.above, d);
            }
            if (lane == 0) sh_warp[warp] = st;
        }
        __syncthreads();
        if (tid == 0) {
            float m = sh_warp[0].m;
            for (int w = 1; w < kWarps; ++w) m = fmaxf(m, sh_warp[w].m);
            Stats sum = {m, 0.0f, 0.0f, 0u};
            for (int w = 0; w < kWarps; ++w) {
                Stats p = sh_warp[w];
                p.move(m, c);
                sum.z += p.z;
                sum.s += p.s;
                sum.above += p.above;
            }
            sh_part = sum;
        }

        // ---- this part's alternatives ----
        if constexpr (TOP) {
            unsigned n = sh_count;
            const unsigned need = min(static_cast<unsigned>(a.top_n), c_hi - c_lo);
            bool strict = !(floor > -INFINITY);          // the list holds what is above the floor, not what equals it
            if (n > static_cast<unsigned>(kCap) && !strict) {
                __syncthreads();                         // everyone has read the count
                if (tid == 0) sh_count = 0;
                __syncthreads();
                gather_above<DTYPE, SCHEME>(a, row, c_lo, c_hi, floor, sh_list, &sh_count);
                __syncthreads();
                n = sh_count;
                strict = true;
            }
            for (unsigned i = tid; i < static_cast<unsigned>(kMaxTop); i += kThreads) sh_top[i] = 0;
            __syncthreads();
            if (n <= static_cast<unsigned>(kCap)) {
                for (unsigned i = tid; i < n; i += kThreads) {
                    const uint64_t mine = sh_list[i];
                    unsigned rank = 0;
#pragma unroll 4
                    for (unsigned o = 0; o < n; ++o) rank += sh_list[o] > mine ? 1u : 0u;
                    if (rank < need) sh_top[rank] = mine;
                }
                if (n < need && warp == 0) fill_equal<DTYPE, SCHEME>(a, row, c_lo, c_hi, floor, sh_top, n, need);
            } else {
                select_rounds<DTYPE, SCHEME>(a, row, c_lo, c_hi, sh_top, need, sh_scratch);
            }
        }
        __syncthreads();

        // ---- the row ----
        cluster.sync();
        if (part == 0) {
            double z = 0.0, s = 0.0;
            uint32_t above = 0;
            float m = sh_part.m;
            for (unsigned r = 1; r < parts; ++r) m = fmaxf(m, cluster.map_shared_rank(&sh_part, r)->m);
            for (unsigned r = 0; r < parts; ++r) {
                Stats p = *cluster.map_shared_rank(&sh_part, r);
                p.move(m, c);
                z += static_cast<double>(p.z);
                s += static_cast<double>(p.s);
                above += p.above;
            }
            const bool nothing = z == 0.0;               // every logit is -inf
            const double ln_z = log(z);
            const double inv_tau = 1.0 / a.tau;
            auto logp = [&](float x) -> float {
                if (nothing) return -INFINITY;
                return static_cast<float>((static_cast<double>(x) - static_cast<double>(m)) * inv_tau - ln_z);
            };
            if (tid == 0) {
                if (a.out_logprob) a.out_logprob[row] = logp(xt);
                if (a.out_entropy)
                    a.out_entropy[row] = nothing ? 0.0f : static_cast<float>(ln_z - 0.6931471805599453 * s / z);
                if (a.out_rank) a.out_rank[row] = 1 + static_cast<int32_t>(above);
                const bool bad = z != z;                 // a NaN or +inf among the logits
                if (a.out_max) a.out_max[row] = bad ? NAN : nothing ? -INFINITY : m;
                if (a.out_sumexp) a.out_sumexp[row] = static_cast<float>(z);
            }
            if constexpr (TOP) {
                const unsigned n = a.top_n, all = n * parts;
                for (unsigned i = tid; i < all; i += kThreads) sh_all[i] = cluster.map_shared_rank(&sh_top[0], i / n)[i % n];
                for (unsigned i = tid; i < n; i += kThreads) {       // places no column takes
                    if (i >= V) {
                        if (a.out_top_ids) a.out_top_ids[row * n + i] = -1;
                        if (a.out_top_logprobs) a.out_top_logprobs[row * n + i] = -INFINITY;
                    }
                }
                __syncthreads();
                for (unsigned i = tid; i < all; i += kThreads) {
                    const uint64_t mine = sh_all[i];
                    if (mine == 0) continue;
                    unsigned rank = 0;
                    if (parts == 1) rank = i;
                    else
                        for (unsigned o = 0; o < all; ++o) rank += sh_all[o] > mine ? 1u : 0u;
                    if (rank < n) {
                        if (a.out_top_ids) a.out_top_ids[row * n + rank] = static_cast<int32_t>(0xFFFFFFFFu - static_cast<uint32_t>(mine));
                        if (a.out_top_logprobs) a.out_top_logprobs[row * n + rank] = logp(composite_value(mine));
                    }
                }
            }
        }
        cluster.sync();                                  // the other parts' shared memory has been read
    }
}

// Gradient: no reduction, so a row is cut into blocks of kGradVectors vectors per thread and every
// block works alone.
constexpr int kGradThreads = 256;
constexpr int kGradVectors = 4;

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
    __device__ __forceinline__ float at(float l, uint32_t col) const {
        const float x = max_nan((l - m) * c, kFar);
        const float g = -ex2_approx_ftz(x) * fmaf(slope, x, base);
        return col == t ? g + own : g;
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
    GradRow r = {0.0f, a.c, 0.0f, 0.0f, 0.0f, 0xFFFFFFFFu};
    bool zero = padded;
    if (!padded) {
        const double z = a.sumexp[row];
        if (z == 0.0) {                                  // every logit is -inf: nothing to move
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
    RowSeedS<SCHEME> rs;
    if (!zero) rs.init(a.bias.key, a.ctx + row * a.W, a.W);

    const uint32_t first = block * (kGradThreads * kGradVectors) + threadIdx.x;
    uint4 w[kGradVectors];
    if (!zero) {
#pragma unroll
        for (int u = 0; u < kGradVectors; ++u) {
            const uint32_t j = first + u * kGradThreads;
            if (j < layout.nvec) w[u] = load_vector_rw(vectors + j);
        }
    }
#pragma unroll
    for (int u = 0; u < kGradVectors; ++u) {
        const uint32_t j = first + u * kGradThreads;
        if (j >= layout.nvec) break;
        const uint32_t col = layout.head + j * VEC;
        float g[VEC];
        if (zero) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) g[i] = 0.0f;
        } else {
            bias_vector<DTYPE, SCHEME>(w[u], rs, a.vocab_offset + col, a.bias);
#pragma unroll
            for (int i = 0; i < VEC; ++i) g[i] = r.at(element<DTYPE>(w[u], i), col + i);
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
            reinterpret_cast<uint4 *>(out_vectors)[j] = o;
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) store_one<DTYPE>(out_ptr, col + i, g[i]);
        }
    }
    if (block == 0) {                                    // ragged ends
        const uint32_t first_tail = layout.head + layout.nvec * VEC;
        uint32_t col = V;
        if (threadIdx.x < layout.head) col = threadIdx.x;
        else if (threadIdx.x >= 32 && threadIdx.x - 32 < V - first_tail) col = first_tail + threadIdx.x - 32;
        if (col < V)
            store_one<DTYPE>(out_ptr, col, zero ? 0.0f : r.at(biased_at<DTYPE, SCHEME>(row_ptr, col, rs, a.vocab_offset + col, a.bias), col));
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
    if (!(c > 1e-30 && c < 1e23)) return SBW_ERR_INVALID_ARG;      // temperature too small or too large for fp32 exponents
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

template <int DTYPE, int SCHEME, bool TOP>
int launch_logprobs(const LogprobArgs &a, cudaStream_t s) {
    DeviceInfo di;
    if (int rc = current_device_info(&di)) return rc;
    const int64_t resident = static_cast<int64_t>(di.sm_count) * (SCHEME == kSchemeNone ? 2 : 1);
    int parts = 1;
    while (parts < kMaxCluster && a.B * parts * 2 <= resident && a.V >= 4096 * parts) parts *= 2;
    cudaLaunchConfig_t cfg = {};
    const int64_t ctas = parts > 1 ? a.B * parts : (a.B < resident ? a.B : resident);
    cfg.gridDim = dim3(static_cast<unsigned>(ctas));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(parts);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    SBW_CUDA_TRY(cudaLaunchKernelEx(&cfg, logprob_kernel<DTYPE, SCHEME, TOP>, a));
    return SBW_OK;
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
    a.tau = static_cast<double>(temperature);
    a.c = static_cast<float>(1.4426950408889634 / static_cast<double>(temperature));
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
