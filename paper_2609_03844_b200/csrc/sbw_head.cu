// sbw_head_logits: the projection to the vocabulary on the 5th-generation tensor cores, hidden states and
// weights in e4m3 with one fp32 scale for each block of 128, and the watermark (Eq. 1 + Eq. 2) in its
// epilogue.
//
//     l[b, v] = sum_kb  xs[b, kb] ws[v / 128, kb]  sum_{k in block kb} x[b, k] w[v, k]
//
// Every CTA is persistent and owns an SM: it walks tiles of 128 rows (hidden states) by BN columns
// (vocabulary).
//   warp 0       copies 128-byte wide blocks of both operands into a ring of shared-memory stages (TMA)
//   warp 1       one thread issues tcgen05.mma: the product of one block of 128 goes to one of the
//                accumulators in tensor memory and starts from zero there
//   warps 4..11  read that product back, multiply it by the two scales and add it to fp32 sums in
//                registers: a block's scales are arbitrary fp32 numbers, which the matrix unit cannot
//                apply itself; row = lane, so that a thread's row has one scale per block
// The hidden states are the side with 128 rows whatever B is: at small B the weights' bytes bound the
// call and the matrix unit's time for rows that are not there is hidden behind them.  (With the sides
// exchanged every thread needs a scale per column and block from shared memory.)
//
// Bound: up to 128 rows the weights' bytes, and in repeated calls the 1000 W cap (1 x 128256 x 4096: 109 us, 4.8 TB/s; 90 us, 5.8
// TB/s in short runs, which the cap does not hold back); above, the fp32 sums of the epilogue's warps beside the products
// (2048 x 128256 x 4096: 1.29 ms, 1.10 in short runs; the products alone take 0.65, with the copies 0.77).  There is one
// CTA per tile of 128 or 256 columns and no split along K, so few columns leave SMs idle: 4096 columns for up to 128 rows are 32
// tiles (24 x 4096 x 128256: 357 us, where the bytes take 81), 1000 are 8 (1 x 1000 x 8192: 26 us).
//
// Every wait is bounded: one that does not end within kWaitLimit gives up, the rest of the CTA's logits are NaN, the kernel
// returns, and sbw_head_gave_up tells of it.
#include <atomic>
#include <cuda.h>
#include <cuda_bf16.h>

#include "sbw_common.cuh"
#include "sbw_hash.cuh"
#include "sbw_rowbias.cuh"

namespace sbw {
namespace {

constexpr int kBlock = 128;            // columns of the operands per scale, and bytes per row of a stage
constexpr int kTileM = 128;
constexpr int kHeadThreads = 384;
constexpr int kEpilogueWarps = 8;
constexpr int kMaxStages = 6;                        // of narrow tiles; 4 of wide ones
constexpr int kTmemColumns = 512;
constexpr uint64_t kWaitLimit = 2000000000ull;      // nanoseconds
constexpr uint64_t kLongestLook = 10000000ull;      // more than that between two looks at the clock is time switched out
constexpr int kRowWords = 64;                        // of a row that go through the staging area at a time
constexpr int kRowStride = kRowWords + 2;            // 8-byte accesses by row and by column without bank conflicts; the
                                                     // two words behind a row hold its watermark seed
constexpr int kStagingBytes = kTileM * kRowStride * 4;
constexpr int kMaxDynamicBytes = 227 * 1024 - 1024;  // what a CTA can have less the barriers
// Stages of tiles of n columns beside the staging area and what aligning them takes.
constexpr int stages_of(int n) { return (kMaxDynamicBytes - 1024 - kStagingBytes) / ((n + kTileM) * kBlock); }
static_assert(stages_of(128) == kMaxStages && stages_of(256) == 4, "");

struct HeadArgs {
    const float *xs, *ws;
    int64_t ld_xs, ld_ws;
    void *logits;
    int64_t ld;
    uint32_t B, V, kblocks;
    uint32_t m_tiles;
    int64_t tiles;
    uint32_t x_bytes;          // of one stage's block of hidden states that are copied
    uint32_t stages;
    uint32_t strided;          // rows of the logits do not start on 8-byte boundaries
    const int32_t *ctx;
    int W;
    uint32_t vocab_offset;
    BiasParams bias;
#ifdef SBW_DEBUG
    int64_t stop_at;           // a CTA's products stop at this block, as where a wait ran out
    int64_t withhold_from;     // a CTA's blocks from this one on are not copied, so that the wait for them runs out
    uint64_t wait_limit;
#endif
};

__device__ unsigned long long g_gave_up;   // CTAs in which a wait gave up, since the module was loaded

#ifdef SBW_DEBUG
__device__ __forceinline__ uint64_t wait_limit(const HeadArgs &a) { return a.wait_limit; }
#else
__device__ __forceinline__ uint64_t wait_limit(const HeadArgs &) { return kWaitLimit; }
#endif

// ---- one-line PTX ---------------------------------------------------------------------------

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.b32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
// Waits for the phase of the given parity to end; false if it did not within the limit or, where
// `gave_up` is given, another thread of the CTA gave up.
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, volatile uint32_t *gave_up, uint64_t limit = kWaitLimit) {
    if (barrier_try(bar, parity)) return true;
    uint64_t waited = 0, before = now_ns();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 16; ++i)
            if (barrier_try(bar, parity)) return true;
        if (gave_up && *gave_up) return false;
        const uint64_t now = now_ns();
        waited += min(now - before, kLongestLook);
        before = now;
        if (waited > limit) {
            if (gave_up) *gave_up = 1u;
            return false;
        }
    }
}
__device__ __forceinline__ void copy_block(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// Operand block in shared memory: rows of 128 bytes, 128-byte swizzle, groups of 8 rows 1024 bytes apart.
__device__ __forceinline__ uint64_t operand(uint32_t addr) {
    return static_cast<uint64_t>((addr & 0x3ffffu) >> 4) | uint64_t(1) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 |
           uint64_t(2) << 61;
}
__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t form, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(form), "r"(static_cast<uint32_t>(add)) : "memory");
}
// A load that stays where it is written: the compiler may move an ordinary one behind the wait that it is to overlap.
__device__ __forceinline__ float load_now(const float *p) {
    float v;
    asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// 16 columns of a warp's 32 lanes; the values may be used after read_done on the same array.
__device__ __forceinline__ void read_columns(uint32_t (&r)[16], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(addr));
}
__device__ __forceinline__ void read_done(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}
// Two fp32 operations per instruction.
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair_of(uint32_t a, uint32_t b) {
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "r"(a), "r"(b));
    return p;
}
__device__ __forceinline__ void of_pair(Pair p, uint32_t &a, uint32_t &b) { asm("mov.b64 {%0, %1}, %2;" : "=r"(a), "=r"(b) : "l"(p)); }
__device__ __forceinline__ Pair pair_fma(Pair a, Pair b, Pair c) {
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint32_t bf16_pair(Pair p) {
    uint32_t a, b;
    of_pair(p, a, b);
    const __nv_bfloat162 q = __floats2bfloat162_rn(__uint_as_float(a), __uint_as_float(b));
    return *reinterpret_cast<const uint32_t *>(&q);
}

// ---- the epilogue's last step ---------------------------------------------------------------

// What a row's seed takes to make, as one number.
template <int SCHEME>
__device__ __forceinline__ uint64_t row_seed(const HeadArgs &a, int64_t row) {
    if (!SBW_CHECKED(row >= 0 && row < a.B, SBW_SITE_HEAD_LOAD)) return 0ull;
    if constexpr (SCHEME == SBW_SCHEME_CONTEXT) return seed_context(a.bias.key, a.ctx + row * a.W, a.W);
    else return jenkins_min(a.ctx + row * a.W, a.W);
}

// A scale of a [rows, blocks of 128] array.
__device__ __forceinline__ float load_scale(const HeadArgs &a, const float *p, const float *base, int64_t rows, int64_t ld) {
    if (!SBW_CHECKED(lies_in_rows(p, 1, base, 4, rows, a.kblocks, ld), SBW_SITE_HEAD_LOAD)) return 0.0f;
    return load_now(p);
}

// The green tests of a tile, made by the epilogue's warps while they wait for its products: at small B the weights'
// bytes leave them idle most of the time (64 x 128256 x 4096: 135 us with the tests after the sums).  A warp has every
// eighth row of the tile and a lane COLS columns of each 64 words of it, next to each other or (strided) 32 apart; a test
// is one bit.
template <int DTYPE, int SCHEME, int BN>
struct Greens {
    static constexpr int PER = DTYPE == SBW_DTYPE_F32 ? 1 : 2, COLS = 2 * PER;
    static constexpr int kRows = kTileM / kEpilogueWarps, kParts = BN / PER / kRowWords;
    static constexpr int kBits = kRows * kParts * COLS;
    uint64_t bits[SCHEME == kSchemeNone ? 1 : kBits / 64];
    uint32_t done, steps;

    __device__ __forceinline__ void begin(int rows, int warp) {
#pragma unroll
        for (auto &b : bits) b = 0ull;
        done = 0u;
        steps = rows > warp ? static_cast<uint32_t>((rows - warp + kEpilogueWarps - 1) / kEpilogueWarps) * kParts : 0u;
    }
    // Up to `most` more: step i is part i % kParts of the warp's row i / kParts, whose seed lies behind its place in the
    // staging area.
    __device__ __forceinline__ void advance(const HeadArgs &a, const uint32_t *staging, uint32_t most, uint32_t col0, int warp, int lane) {
        if constexpr (SCHEME != kSchemeNone) {
#pragma unroll 1
            for (; most > 0u && done < steps; --most, ++done) {
                const uint64_t seed = *reinterpret_cast<const uint64_t *>(staging + (warp + done / kParts * kEpilogueWarps) * kRowStride + kRowWords);
                RowSeedS<SCHEME> rs;
                if constexpr (SCHEME == SBW_SCHEME_CONTEXT) rs.rk = make_row_keys(seed);
                else rs.jmin = static_cast<uint32_t>(seed);
                const uint32_t first = a.vocab_offset + col0 + done % kParts * (kRowWords * PER);
                uint32_t x[COLS];
                if (a.strided) {
#pragma unroll
                    for (int i = 0; i < COLS; ++i) x[i] = rs.word0(first + 32 * i + lane, a.bias.key, a.bias.weyl);
                } else {
                    rs.template word0_n<COLS>(first + lane * COLS, a.bias.key, a.bias.weyl, x);
                }
                uint64_t g = 0;
#pragma unroll
                for (int i = 0; i < COLS; ++i) g |= static_cast<uint64_t>(x[i] <= a.bias.thr_m1) << i;
                const uint32_t at = done * COLS;
#pragma unroll
                for (int i = 0; i < kBits / 64; ++i)
                    if (at / 64 == static_cast<uint32_t>(i)) bits[i] |= g << (at % 64);
            }
        }
    }
    // Those of part `part` of the warp's row number r.
    __device__ __forceinline__ uint32_t of(int r, int part) const {
        const uint32_t at = static_cast<uint32_t>(r * kParts + part) * COLS;
        uint64_t b = bits[0];
#pragma unroll
        for (int i = 1; i < kBits / 64; ++i)
            if (at / 64 == static_cast<uint32_t>(i)) b = bits[i];
        return static_cast<uint32_t>(b >> (at % 64));
    }
};

// Writes 64 words (64 fp32 logits, or 128 bf16 ones in pairs) of each of `rows` rows from the staging area, every warp
// each eighth row, a lane two words: a row is one 256-byte store.  Words were laid out there by row = lane.  Eight rows are
// read before the first is stored: the compiler keeps reads behind stores that it cannot tell from them, and one row at a
// time took 150 clocks a row (2048 x 128256 x 4096: 1.3 of 2.1 ms).
template <int DTYPE, int SCHEME, int BN>
__device__ __forceinline__ void store_rows(const HeadArgs &a, const uint32_t *staging, const Greens<DTYPE, SCHEME, BN> &greens, int part,
                                           int rows, int64_t row0, uint32_t col0, int warp, int lane) {
    constexpr int PER = DTYPE == SBW_DTYPE_F32 ? 1 : 2, COLS = 2 * PER, ESIZE = 4 / PER, kAtOnce = 8;
    char *const base = static_cast<char *>(a.logits) + (row0 * a.ld + col0) * ESIZE;
    const int64_t stride = a.ld * ESIZE;
#pragma unroll 1
    for (int i0 = 0; warp + i0 * kEpilogueWarps < rows; i0 += kAtOnce) {
        uint2 w[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int r = warp + (i0 + u) * kEpilogueWarps;
            const uint32_t *const from = staging + r * kRowStride;
            if (r >= rows) {
                w[u] = make_uint2(0u, 0u);
            } else if (!a.strided) {
                w[u] = *reinterpret_cast<const uint2 *>(from + 2 * lane);
            } else if constexpr (DTYPE == SBW_DTYPE_F32) {
                w[u] = make_uint2(from[lane], from[32 + lane]);
            } else {
                const uint16_t *const e = reinterpret_cast<const uint16_t *>(from);
                w[u] = make_uint2(e[lane] | static_cast<uint32_t>(e[32 + lane]) << 16, e[64 + lane] | static_cast<uint32_t>(e[96 + lane]) << 16);
            }
        }
        if constexpr (SCHEME != kSchemeNone) {
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const uint32_t g = greens.of(i0 + u, part);
                if constexpr (DTYPE == SBW_DTYPE_F32) {
                    if (g & 1u) w[u].x = __float_as_uint(__fadd_rn(__uint_as_float(w[u].x), a.bias.delta));
                    if (g & 2u) w[u].y = __float_as_uint(__fadd_rn(__uint_as_float(w[u].y), a.bias.delta));
                } else {
                    const uint32_t lo = a.bias.delta_bf16, hi = a.bias.delta_bf16 << 16;
                    w[u].x = add_bf16x2(w[u].x, (g & 1u ? lo : 0x8000u) | (g & 2u ? hi : 0x80000000u));
                    w[u].y = add_bf16x2(w[u].y, (g & 4u ? lo : 0x8000u) | (g & 8u ? hi : 0x80000000u));
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int r = warp + (i0 + u) * kEpilogueWarps;
            if (r >= rows) break;
            (void)SBW_CHECKED(r < kTileM, SBW_SITE_HEAD_SHARED);
            char *const at = base + r * stride;
            const uint32_t first = a.strided ? lane : lane * COLS, apart = a.strided ? 32 : 1;
            if (!a.strided && col0 + first + COLS <= a.V) {
                if (SBW_CHECKED(lies_in_rows(at + lane * 8, COLS, a.logits, ESIZE, a.B, a.V, a.ld), SBW_SITE_HEAD_STORE))
                    *reinterpret_cast<uint2 *>(at + lane * 8) = w[u];
            } else {
#pragma unroll
                for (int i = 0; i < COLS; ++i) {
                    const uint32_t v = i < PER ? w[u].x : w[u].y, c = first + i * apart;
                    if (col0 + c >= a.V || !SBW_CHECKED(lies_in_rows(at + c * ESIZE, 1, a.logits, ESIZE, a.B, a.V, a.ld), SBW_SITE_HEAD_STORE)) break;
                    if constexpr (DTYPE == SBW_DTYPE_F32) reinterpret_cast<uint32_t *>(at)[c] = v;
                    else reinterpret_cast<uint16_t *>(at)[c] = static_cast<uint16_t>(v >> (16 * (i & 1)));
                }
            }
        }
    }
}

template <int DTYPE, int SCHEME, int BN>
__global__ void __launch_bounds__(kHeadThreads, 1)
    head_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const HeadArgs a) {
    constexpr int PART = BN / 2;                       // columns of one warpgroup of the epilogue
    constexpr int NBUF = kTmemColumns / BN;            // accumulators
    constexpr uint32_t kWBytes = BN * kBlock;
    // fp32 accumulator, both operands e4m3 with K along their rows, 128 x BN
    constexpr uint32_t kForm = 1u << 4 | static_cast<uint32_t>(BN / 8) << 17 | static_cast<uint32_t>(kTileM / 16) << 24;
    extern __shared__ uint8_t dynamic_smem[];
    __shared__ __align__(8) uint64_t bars[2 * kMaxStages + 2 * NBUF + 1];
    __shared__ uint32_t tmem_slot;
    __shared__ uint32_t gave_up_slot;
    volatile uint32_t *const gave_up = &gave_up_slot;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t stages_at = (smem_addr(dynamic_smem) + 1023u) & ~1023u;
    const uint32_t stage_bytes = kWBytes + kTileM * kBlock, copied = kWBytes + a.x_bytes;
    uint32_t *const staging = reinterpret_cast<uint32_t *>(
        dynamic_smem + (stages_at - smem_addr(dynamic_smem)) + a.stages * stage_bytes);
    (void)SBW_CHECKED(lies_in_shared(staging, kStagingBytes, dynamic_smem), SBW_SITE_HEAD_SHARED);
    const uint32_t full = smem_addr(bars), empty = full + 8 * kMaxStages;
    const uint32_t ready = empty + 8 * kMaxStages, taken = ready + 8 * NBUF, last = taken + 8 * NBUF;

    // Rows of hidden states that are not there are 0 in every stage: the matrix unit multiplies 128 rows whatever B is, and
    // other bytes in their place cost power and so clocks (B = 1, 128256 x 4096 back to back: 114 us with the next stage's
    // bytes there and 11 stages, 109 with zeros and 6).
    if (a.x_bytes < kTileM * kBlock) {
        uint8_t *const all = dynamic_smem + (stages_at - smem_addr(dynamic_smem));
        for (uint32_t s = 0; s < a.stages; ++s)
            for (uint32_t i = a.x_bytes + threadIdx.x * 16; i < kTileM * kBlock; i += kHeadThreads * 16)
                *reinterpret_cast<uint4 *>(all + s * stage_bytes + kWBytes + i) = make_uint4(0u, 0u, 0u, 0u);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < kMaxStages; ++i) {
            barrier_init(full + 8 * i, 1);
            barrier_init(empty + 8 * i, 1);
        }
        for (uint32_t i = 0; i < NBUF; ++i) {
            barrier_init(ready + 8 * i, 1);
            barrier_init(taken + 8 * i, kEpilogueWarps);
        }
        barrier_init(last, 1);
        gave_up_slot = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_slot)),
                     "r"(kTmemColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_slot;
    int64_t issued = 0;                                  // by thread 0: blocks copied
    const uint64_t limit = wait_limit(a);
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // The epilogue's warps take more registers than an even share (64 x 128256 x 4096 watermarked: 162 us without, 145 with
    // it).  The split is the whole of what the launch has, which launch_head checks: a warpgroup would wait for good for
    // registers that are not there.
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 0 && lane == 0) {
            uint32_t stage = 0, parity = 0;
            bool ok = true;
            for (int64_t t = blockIdx.x; ok && t < a.tiles; t += gridDim.x) {
                const int m0 = static_cast<int>(t % a.m_tiles) * kTileM, v0 = static_cast<int>(t / a.m_tiles) * BN;
                for (uint32_t kb = 0; kb < a.kblocks; ++kb) {
#ifdef SBW_DEBUG
                    if (issued == a.withhold_from) {
                        ok = false;
                        break;
                    }
#endif
                    ok = barrier_wait(empty + 8 * stage, parity ^ 1u, gave_up, limit);
                    if (!ok) break;
                    const uint32_t at = stages_at + stage * stage_bytes;
                    barrier_expect(full + 8 * stage, copied);
                    copy_block(at, &map_w, static_cast<int>(kb) * kBlock, v0, full + 8 * stage);
                    copy_block(at + kWBytes, &map_x, static_cast<int>(kb) * kBlock, m0, full + 8 * stage);
                    ++issued;
                    if (++stage == a.stages) {
                        stage = 0;
                        parity ^= 1u;
                    }
                }
            }
            // Copies in flight have to land before the CTA's shared memory goes.  Where the products stopped nobody else has
            // waited for the last ones, whether this thread gave up or had issued everything by then.
            for (uint32_t i = 0; i < a.stages && i < issued; ++i) {
                const int64_t n = issued - 1 - i;
                if (!barrier_wait(full + 8 * static_cast<uint32_t>(n % a.stages), static_cast<uint32_t>(n / a.stages) & 1u, nullptr))
                    *gave_up = 1u;
            }
        } else if (warp == 1 && lane == 0) {
            uint32_t stage = 0, parity = 0, buf = 0, buf_parity = 0;
            bool ok = true;
#ifdef SBW_DEBUG
            int64_t block = 0;
#endif
            for (int64_t t = blockIdx.x; ok && t < a.tiles; t += gridDim.x) {
                for (uint32_t kb = 0; kb < a.kblocks; ++kb) {
#ifdef SBW_DEBUG
                    if (block++ == a.stop_at) {
                        for (const uint64_t start = now_ns(); now_ns() - start < 1000000ull;) {}      // products under way end first
                        *gave_up = 1u;
                        ok = false;
                        break;
                    }
#endif
                    ok = barrier_wait(taken + 8 * buf, buf_parity ^ 1u, gave_up, limit) &&
                         barrier_wait(full + 8 * stage, parity, gave_up, limit);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t at = stages_at + stage * stage_bytes;
                    const uint64_t x = operand(at + kWBytes), w = operand(at);
#pragma unroll
                    for (int k = 0; k < 4; ++k)        // 32 of a block's 128 at a time: 32 bytes further on in every row
                        multiply(tmem + buf * BN, x + 2 * k, w + 2 * k, kForm, k > 0);
                    commit(empty + 8 * stage);
                    commit(ready + 8 * buf);
                    if (++stage == a.stages) {
                        stage = 0;
                        parity ^= 1u;
                    }
                    if (++buf == NBUF) {
                        buf = 0;
                        buf_parity ^= 1u;
                    }
                }
            }
            commit(last);                              // no product is in flight when the tensor memory goes
            if (!barrier_wait(last, 0u, nullptr)) *gave_up = 1u;
        }
        __syncwarp();
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        const int quarter = warp % 4, wg = warp / 4 - 1;
        uint32_t buf = 0, parity = 0;
        int64_t seeds_of = -1;                           // first row of the tile whose seeds are there
        bool ok = true;
        for (int64_t t = blockIdx.x; t < a.tiles; t += gridDim.x) {
            const int64_t row0 = (t % a.m_tiles) * kTileM + quarter * 32;
            const uint32_t col0 = static_cast<uint32_t>(t / a.m_tiles) * BN + wg * PART;
            const int64_t left = static_cast<int64_t>(a.B) - row0;
            const int rows = left < 0 ? 0 : left < 32 ? static_cast<int>(left) : 32;
            const int64_t row = row0 + (lane < rows ? lane : 0);
            const uint32_t vb = min(col0, a.V - 1) / kBlock;
            const float *const ws = a.ws + static_cast<int64_t>(vb) * a.ld_ws;
            const float *const xs = a.xs + (rows ? row : 0) * a.ld_xs;
            const int64_t m0 = (t % a.m_tiles) * kTileM;
            const int tile_rows = static_cast<int64_t>(a.B) - m0 < kTileM ? static_cast<int>(a.B - m0) : kTileM;
            const uint32_t tile_col = static_cast<uint32_t>(t / a.m_tiles) * BN;
            Greens<DTYPE, SCHEME, BN> greens;
            greens.begin(tile_rows, warp - 4);
            if constexpr (SCHEME != kSchemeNone) {
                if (m0 != seeds_of) {                    // the rows' seeds, behind their places in the staging area
                    if (wg == 0 && rows)
                        *reinterpret_cast<uint64_t *>(staging + (quarter * 32 + lane) * kRowStride + kRowWords) = row_seed<SCHEME>(a, row);
                    asm volatile("bar.sync 1, 256;" ::: "memory");
                    seeds_of = m0;
                }
            }
            const uint32_t per_block = SCHEME == kSchemeNone ? 0u : (greens.steps + a.kblocks - 1) / a.kblocks;
            Pair acc[PART / 2];
#pragma unroll
            for (int i = 0; i < PART / 2; ++i) acc[i] = 0ull;
            const int64_t w_rows = (static_cast<int64_t>(a.V) + kBlock - 1) / kBlock;
            float sx = load_scale(a, xs, a.xs, a.B, a.ld_xs), sw = load_scale(a, ws, a.ws, w_rows, a.ld_ws);    // a block's scales are on their way while the one before is added
            for (uint32_t kb = 0; kb < a.kblocks; ++kb) {
                const float s = sx * sw;
                if (kb + 1 < a.kblocks) {
                    sx = load_scale(a, xs + kb + 1, a.xs, a.B, a.ld_xs);
                    sw = load_scale(a, ws + kb + 1, a.ws, w_rows, a.ld_ws);
                }
                greens.advance(a, staging, per_block, tile_col, warp - 4, lane);
                if (ok) ok = __all_sync(0xffffffffu, barrier_wait(ready + 8 * buf, parity, gave_up, limit));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t from = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + buf * BN + wg * PART;
                const Pair both = pair_of(__float_as_uint(s), __float_as_uint(s));
                uint32_t r[2][16];
                if (rows) read_columns(r[0], from);
#pragma unroll
                for (int c = 0; c < PART / 16; ++c) {
                    if (rows) {
                        read_done(r[c & 1]);
                        if (c + 1 < PART / 16) read_columns(r[(c + 1) & 1], from + 16 * (c + 1));
                    }
                    if (c + 1 == PART / 16) {
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) barrier_arrive(taken + 8 * buf);
                    }
                    if (rows) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            acc[8 * c + i] = pair_fma(pair_of(r[c & 1][2 * i], r[c & 1][2 * i + 1]), both, acc[8 * c + i]);
                    }
                }
                if (++buf == NBUF) {
                    buf = 0;
                    parity ^= 1u;
                }
            }
            if (!ok) {
#pragma unroll
                for (int i = 0; i < PART / 2; ++i) acc[i] = ~0ull;           // NaN
            }
            // The sums leave through the staging area, 64 words of a row at a time: all or half of the columns of
            // one warpgroup, or those of both.
            constexpr int PER = DTYPE == SBW_DTYPE_F32 ? 1 : 2;
            constexpr int kOwnWords = PART / PER, WORDS = kOwnWords < kRowWords ? kOwnWords : kRowWords;
            constexpr int kTogether = kRowWords / WORDS, kSub = kOwnWords / WORDS, kPasses = 2 * kOwnWords / kRowWords;
#pragma unroll
            for (int pass = 0; pass < kPasses; ++pass) {
                if (rows && (kTogether > 1 ? wg / kTogether == pass : wg == pass / kSub)) {
                    uint32_t *const to = staging + (quarter * 32 + lane) * kRowStride + wg % kTogether * WORDS;
                    (void)SBW_CHECKED(lies_in_shared(to, WORDS * 4, dynamic_smem), SBW_SITE_HEAD_SHARED);
#pragma unroll
                    for (int i = 0; i < WORDS; i += 2) {
                        uint2 w;
                        if constexpr (DTYPE == SBW_DTYPE_F32) of_pair(acc[(i + pass % kSub * WORDS) / 2], w.x, w.y);
                        else w = make_uint2(bf16_pair(acc[i + pass % kSub * WORDS]), bf16_pair(acc[i + 1 + pass % kSub * WORDS]));
                        *reinterpret_cast<uint2 *>(to + i) = w;
                    }
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
                store_rows<DTYPE, SCHEME, BN>(a, staging, greens, pass, tile_rows, m0, tile_col + pass * kRowWords * PER, warp - 4, lane);
                asm volatile("bar.sync 1, 256;" ::: "memory");
            }
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0 && *gave_up) atomicAdd(&g_gave_up, 1ull);
#ifdef SBW_DEBUG
    if (threadIdx.x == 0)
        for (int64_t n = issued - 1; n >= 0 && n >= issued - a.stages; --n)
            (void)SBW_CHECKED(barrier_try(full + 8 * static_cast<uint32_t>(n % a.stages), static_cast<uint32_t>(n / a.stages) & 1u),
                              SBW_SITE_HEAD_COPY);
#endif
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemColumns) : "memory");
    }
}

// ---- host -----------------------------------------------------------------------------------

#ifdef SBW_DEBUG
std::atomic<int64_t> debug_stop_at{-1}, debug_withhold_from{-1};
std::atomic<uint64_t> debug_wait_limit{kWaitLimit};
#endif

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int encode_entry(EncodeTiled *out) {
    static std::atomic<void *> found{nullptr};
    void *p = found.load(std::memory_order_acquire);
    if (!p) {
        cudaDriverEntryPointQueryResult status;
        SBW_CUDA_TRY(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &status));
        if (status != cudaDriverEntryPointSuccess || !p) return SBW_ERR_UNSUPPORTED;
        found.store(p, std::memory_order_release);
    }
    *out = reinterpret_cast<EncodeTiled>(p);
    return SBW_OK;
}

// A [rows, K] operand copied in blocks of box_rows rows by 128 bytes; what lies outside reads as 0.
int make_map(CUtensorMap *map, const void *p, int64_t rows, int64_t K, int64_t ld, int box_rows) {
    EncodeTiled encode;
    if (int rc = encode_entry(&encode)) return rc;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(K), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld)};
    const cuuint32_t box[2] = {kBlock, static_cast<cuuint32_t>(box_rows)}, unit[2] = {1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(p), dims, strides, box, unit,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return cuda_fail(cudaErrorInvalidValue);
    return SBW_OK;
}

template <int DTYPE, int SCHEME, int BN>
int launch_head(HeadArgs &a, const void *x, int64_t ld_x, const void *w, int64_t ld_w, int64_t K, cudaStream_t stream) {
    DeviceInfo di;
    if (int rc = current_device_info(&di)) return rc;
    const int box_m = a.B < kTileM ? static_cast<int>((a.B + 7) / 8 * 8) : kTileM;
    a.x_bytes = static_cast<uint32_t>(box_m) * kBlock;
    const uint32_t stage_bytes = BN * kBlock + kTileM * kBlock;
    a.stages = stages_of(BN);
    const size_t bytes = 1024 + a.stages * stage_bytes + kStagingBytes;
    a.m_tiles = (a.B + kTileM - 1) / kTileM;
    constexpr int kEsize = DTYPE == SBW_DTYPE_F32 ? 4 : 2;
    a.strided = reinterpret_cast<uintptr_t>(a.logits) % 8 != 0 || a.ld * kEsize % 8 != 0;
    a.tiles = static_cast<int64_t>(a.m_tiles) * ((a.V + BN - 1) / BN);
    CUtensorMap map_x, map_w;
    if (int rc = make_map(&map_x, x, a.B, K, ld_x, box_m)) return rc;
    if (int rc = make_map(&map_w, w, a.V, K, ld_w, BN)) return rc;
    const auto kernel = head_kernel<DTYPE, SCHEME, BN>;
    static std::atomic<uint64_t> prepared{0};
    if (!(prepared.load(std::memory_order_acquire) >> di.device & 1)) {
#ifndef SBW_DEBUG   // separate compilation, as the bounds-flag build has it, leaves the split out
        cudaFuncAttributes f;
        SBW_CUDA_TRY(cudaFuncGetAttributes(&f, kernel));
        if (f.numRegs * kHeadThreads < 40 * 128 + 232 * 256) return SBW_ERR_UNSUPPORTED;
#endif
        SBW_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxDynamicBytes));
        prepared.fetch_or(uint64_t(1) << di.device, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.tiles < di.sm_count ? a.tiles : di.sm_count));
    cfg.blockDim = dim3(kHeadThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    SBW_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, map_x, map_w, a));
    return SBW_OK;
}

template <int DTYPE, int SCHEME>
int launch_head(HeadArgs &a, const void *x, int64_t ld_x, const void *w, int64_t ld_w, int64_t K, cudaStream_t s) {
    // up to 128 rows the weights' bytes bound the call and narrower tiles share them out more evenly;
    // above, each byte of a wider tile's weights serves more products
    return a.B <= kTileM ? launch_head<DTYPE, SCHEME, 128>(a, x, ld_x, w, ld_w, K, s)
                         : launch_head<DTYPE, SCHEME, 256>(a, x, ld_x, w, ld_w, K, s);
}

}  // namespace
}  // namespace sbw

extern "C" int sbw_head_logits(const void *x, int64_t ld_x, const float *x_scales, int64_t ld_x_scales, const void *w,
                               int64_t ld_w, const float *w_scales, int64_t ld_w_scales, int64_t B, int64_t V, int64_t K,
                               void *logits, int dtype, int64_t ld, int64_t vocab_offset, const int32_t *ctx_tokens,
                               int ctx_width, uint64_t key, double gamma, float delta, int scheme, void *stream) {
    using namespace sbw;
    if (!valid_common(dtype, ctx_width, gamma, scheme)) return SBW_ERR_INVALID_ARG;
    if (B < 0 || V <= 0 || K <= 0 || ld < V || vocab_offset < 0) return SBW_ERR_INVALID_ARG;
    if (!(delta == delta) || delta - delta != 0.0f) return SBW_ERR_INVALID_ARG;
    constexpr int64_t kMost = 0x7fffffffLL - 256;           // coordinates of the copies are 32-bit
    if (B > kMost || V > kMost || K > kMost || vocab_offset + V > (int64_t(1) << 32)) return SBW_ERR_UNSUPPORTED;
    const int64_t kblocks = (K + kBlock - 1) / kBlock;
    if (ld_x < K || ld_w < K || ld_x_scales < kblocks || ld_w_scales < kblocks) return SBW_ERR_INVALID_ARG;
    if (B == 0) return SBW_OK;
    const float in_precision = dtype == SBW_DTYPE_BF16 ? __bfloat162float(__float2bfloat16_rn(delta)) : delta;
    const bool marked = in_precision != 0.0f;
    if (!x || !x_scales || !w || !w_scales || !logits || (marked && !ctx_tokens)) return SBW_ERR_INVALID_ARG;
    // operands are copied by tensor maps: 16-byte aligned rows
    if (reinterpret_cast<uintptr_t>(x) % 16 != 0 || reinterpret_cast<uintptr_t>(w) % 16 != 0) return SBW_ERR_INVALID_ARG;
    if ((B > 1 && ld_x % 16 != 0) || (V > 1 && ld_w % 16 != 0)) return SBW_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(x_scales) % 4 != 0 || reinterpret_cast<uintptr_t>(w_scales) % 4 != 0 ||
        reinterpret_cast<uintptr_t>(logits) % (dtype == SBW_DTYPE_F32 ? 4 : 2) != 0)
        return SBW_ERR_INVALID_ARG;
    if (B == 1) ld_x = (K + 15) / 16 * 16;
    if (V == 1) ld_w = (K + 15) / 16 * 16;
    if (ld_x >= (int64_t(1) << 40) || ld_w >= (int64_t(1) << 40)) return SBW_ERR_UNSUPPORTED;
    HeadArgs a = {};
    a.xs = x_scales;
    a.ws = w_scales;
    a.ld_xs = ld_x_scales;
    a.ld_ws = ld_w_scales;
    a.logits = logits;
    a.ld = ld;
    a.B = static_cast<uint32_t>(B);
    a.V = static_cast<uint32_t>(V);
    a.kblocks = static_cast<uint32_t>(kblocks);
    a.ctx = ctx_tokens;
    a.W = ctx_width;
    a.vocab_offset = static_cast<uint32_t>(vocab_offset);
    a.bias.key = key;
    a.bias.thr_m1 = threshold_minus_one(gamma);
    a.bias.delta = in_precision;
    a.bias.delta_bf16 = dtype == SBW_DTYPE_BF16 ? static_cast<uint32_t>(__bfloat16_as_ushort(__float2bfloat16_rn(delta))) : 0u;
    a.bias.weyl = make_weyl();
#ifdef SBW_DEBUG
    a.stop_at = debug_stop_at.load();
    a.withhold_from = debug_withhold_from.load();
    a.wait_limit = debug_wait_limit.load();
#endif
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == SBW_DTYPE_F32) {
        if (!marked) return launch_head<SBW_DTYPE_F32, kSchemeNone>(a, x, ld_x, w, ld_w, K, s);
        return scheme == SBW_SCHEME_CONTEXT ? launch_head<SBW_DTYPE_F32, SBW_SCHEME_CONTEXT>(a, x, ld_x, w, ld_w, K, s)
                                            : launch_head<SBW_DTYPE_F32, SBW_SCHEME_SELFSALT>(a, x, ld_x, w, ld_w, K, s);
    }
    if (!marked) return launch_head<SBW_DTYPE_BF16, kSchemeNone>(a, x, ld_x, w, ld_w, K, s);
    return scheme == SBW_SCHEME_CONTEXT ? launch_head<SBW_DTYPE_BF16, SBW_SCHEME_CONTEXT>(a, x, ld_x, w, ld_w, K, s)
                                        : launch_head<SBW_DTYPE_BF16, SBW_SCHEME_SELFSALT>(a, x, ld_x, w, ld_w, K, s);
}

extern "C" int sbw_head_gave_up(uint64_t *out_ctas, void *stream) {
    using namespace sbw;
    if (!out_ctas) return SBW_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaStreamCaptureStatus capture;
    SBW_CUDA_TRY(cudaStreamIsCapturing(s, &capture));
    if (capture != cudaStreamCaptureStatusNone) return SBW_ERR_UNSUPPORTED;
    unsigned long long ctas = 0;
    SBW_CUDA_TRY(cudaMemcpyFromSymbolAsync(&ctas, g_gave_up, sizeof(ctas), 0, cudaMemcpyDeviceToHost, s));
    SBW_CUDA_TRY(cudaStreamSynchronize(s));
    *out_ctas = ctas;
    return SBW_OK;
}

#ifdef SBW_DEBUG
// Bounds-flag build only: from the next call on, waits inside a CTA give up after limit_ns, and blocks from number
// `withhold_from` of every CTA on (below 0: none) are not copied, so that the wait for them runs out.
extern "C" int sbw_debug_head_waits(uint64_t limit_ns, int64_t withhold_from) {
    sbw::debug_wait_limit.store(limit_ns);
    sbw::debug_withhold_from.store(withhold_from);
    return SBW_OK;
}

// Bounds-flag build only: from the next call on, every CTA's products stop at its block number `block` (counted over its tiles),
// as they do where a wait ran out; below 0 they do not.
extern "C" int sbw_debug_head_stop(int64_t block) {
    sbw::debug_stop_at.store(block);
    return SBW_OK;
}
#endif
