// sbw_quantize_fp8: values to e4m3 codes with one fp32 scale for each block of 128 columns, the form
// in which sbw_head_logits takes hidden states (blocks of one row) and weights (blocks of 128 rows).
//
//     scale = max(amax / 448, 2^-126)       448 = the largest finite e4m3 value
//     code  = e4m3(x / scale)               both quotients correctly rounded fp32, the code to nearest even
//
// One pass: a block's elements stay in registers between the maximum and the division, so every
// element is read once and every code written once (128256 x 4096 bf16 in 128 x 128 blocks, repeated calls: 324 us,
// 4.9 TB/s).
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "sbw_common.cuh"

namespace sbw {
namespace {

constexpr int kBlock = 128;
constexpr int kQuantThreads = 256;

struct QuantArgs {
    const void *x;
    int64_t R, K, ld;
    uint8_t *out;
    int64_t ld_out;
    float *scales;
    int64_t ld_scales;
    uint32_t kblocks;
};

// Quotients by one scale, correctly rounded: with r the rounded reciprocal of s and q = x r rounded, the remainder e = q s - x
// is exact and q - e r, rounded once, is the rounded x / s.  Markstein's theorem (IBM J. Res. Dev. 34, 1990) says so for a q
// within one unit in the last place; x r can be one and a half off (Brisebarre, Muller and Raina, IEEE Trans. Comput. 53, 2004,
// treat that case), so all 2^46 pairs of mantissas were tried on the device: none is wrong.  Powers of two change nothing as
// long as nothing underflows, and for a scale from 2^-90 on and a quotient from 2^-11 on (below, every code is 0) the remainder
// does not.  With the remainder this way round a zero keeps its sign: x = -0 has q = -0, e = +0 and -0 - 0 r = -0.
// Three operations where the division takes about ten (128256 x 4096 bf16, repeated calls: 324 us, 365 with it).  For scales
// out of that range, and one that is no number, the division itself.
struct Divisor {
    float s, minus_r;
    bool plain;
    __device__ __forceinline__ explicit Divisor(float scale) : s(scale), minus_r(-1.0f / scale), plain(!(scale >= 0x1p-90f && scale <= 0x1p90f)) {}
    template <bool PLAIN>
    __device__ __forceinline__ float of(float x) const {
        if constexpr (PLAIN) return __fdiv_rn(x, s);
        const float q = __fmul_rn(x, -minus_r);
        return __fmaf_rn(__fmaf_rn(q, s, -x), minus_r, q);
    }
};

template <int DTYPE>
struct Elements {
    static constexpr int VEC = DTYPE == SBW_DTYPE_F32 ? 4 : 8;     // of one 16-byte load
    static constexpr int LANES = kBlock / VEC;                      // threads that hold one row of a block
    uint4 w;
    __device__ __forceinline__ float at(int i) const {
        const uint32_t *e = reinterpret_cast<const uint32_t *>(&w);
        if constexpr (DTYPE == SBW_DTYPE_F32) return __uint_as_float(e[i]);
        else return __uint_as_float((i & 1) ? (e[i >> 1] & 0xffff0000u) : (e[i >> 1] << 16));
    }
    // Elements col .. col + VEC - 1 of a row; those from K on are 0.
    template <bool VECTOR>
    __device__ __forceinline__ void load(const QuantArgs &a, int64_t row, int64_t col) {
        constexpr int ESIZE = 16 / VEC;
        const char *const row_ptr = static_cast<const char *>(a.x) + row * a.ld * ESIZE;
        w = make_uint4(0u, 0u, 0u, 0u);
        if (VECTOR && col + VEC <= a.K) {
            const char *const p = row_ptr + col * ESIZE;
            if (SBW_CHECKED(lies_in_rows(p, VEC, a.x, ESIZE, a.R, a.K, a.ld), SBW_SITE_QUANT_LOAD)) w = __ldcs(reinterpret_cast<const uint4 *>(p));
        } else {
            uint32_t *e = reinterpret_cast<uint32_t *>(&w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const char *const p = row_ptr + (col + i) * ESIZE;
                if (col + i >= a.K || !SBW_CHECKED(lies_in_rows(p, 1, a.x, ESIZE, a.R, a.K, a.ld), SBW_SITE_QUANT_LOAD)) continue;
                if constexpr (DTYPE == SBW_DTYPE_F32) e[i] = *reinterpret_cast<const uint32_t *>(p);
                else e[i >> 1] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(p)) << (16 * (i & 1));
            }
        }
    }
    // Bits of the largest magnitude.  Magnitudes order like their bit patterns, with infinity above
    // every number and NaN above that, so a NaN is not lost as it would be in a float maximum.
    __device__ __forceinline__ uint32_t largest() const {
        const uint32_t *e = reinterpret_cast<const uint32_t *>(&w);
        if constexpr (DTYPE == SBW_DTYPE_F32) {
            return max(max(e[0] & 0x7fffffffu, e[1] & 0x7fffffffu), max(e[2] & 0x7fffffffu, e[3] & 0x7fffffffu));
        } else {
            const uint32_t m = __vmaxu2(__vmaxu2(e[0] & 0x7fff7fffu, e[1] & 0x7fff7fffu),
                                        __vmaxu2(e[2] & 0x7fff7fffu, e[3] & 0x7fff7fffu));
            return max(m >> 16, m & 0xffffu) << 16;
        }
    }
    // Writes the codes of the elements that exist.
    template <bool VECTOR, bool PLAIN>
    __device__ __forceinline__ void store(const QuantArgs &a, int64_t row, int64_t col, const Divisor &d) const {
        uint8_t *const row_out = a.out + row * a.ld_out;
        uint32_t code[VEC / 4];
#pragma unroll
        for (int i = 0; i < VEC / 4; ++i) {
            const __nv_fp8x2_storage_t lo = __nv_cvt_float2_to_fp8x2(
                make_float2(d.of<PLAIN>(at(4 * i)), d.of<PLAIN>(at(4 * i + 1))), __NV_SATFINITE, __NV_E4M3);
            const __nv_fp8x2_storage_t hi = __nv_cvt_float2_to_fp8x2(
                make_float2(d.of<PLAIN>(at(4 * i + 2)), d.of<PLAIN>(at(4 * i + 3))), __NV_SATFINITE, __NV_E4M3);
            code[i] = static_cast<uint32_t>(lo) | static_cast<uint32_t>(hi) << 16;
        }
        if (VECTOR && col + VEC <= a.K) {
            if (!SBW_CHECKED(lies_in_rows(row_out + col, VEC, a.out, 1, a.R, a.K, a.ld_out), SBW_SITE_QUANT_STORE)) return;
            if constexpr (VEC == 8) *reinterpret_cast<uint2 *>(row_out + col) = make_uint2(code[0], code[1]);
            else *reinterpret_cast<uint32_t *>(row_out + col) = code[0];
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (col + i < a.K && SBW_CHECKED(lies_in_rows(row_out + col + i, 1, a.out, 1, a.R, a.K, a.ld_out), SBW_SITE_QUANT_STORE))
                    row_out[col + i] = static_cast<uint8_t>(code[i >> 2] >> (8 * (i & 3)));
        }
    }
};

__device__ __forceinline__ float scale_of(uint32_t amax_bits) {
    const float s = __fdiv_rn(__uint_as_float(amax_bits), 448.0f);
    return s < 0x1p-126f ? 0x1p-126f : s;       // a NaN stays one
}

__device__ __forceinline__ void store_scale(const QuantArgs &a, int64_t row, uint32_t kb, float s, int block_rows) {
    float *const p = a.scales + row * a.ld_scales + kb;
    if (SBW_CHECKED(lies_in_rows(p, 1, a.scales, 4, (a.R + block_rows - 1) / block_rows, a.kblocks, a.ld_scales), SBW_SITE_QUANT_STORE)) *p = s;
}

// Blocks of one row: LANES threads per block, kUnroll blocks at a time so that as many loads are in
// flight.  Block numbers run along a row first.
template <int DTYPE, bool VECTOR>
__global__ void __launch_bounds__(kQuantThreads) quantize_rows_kernel(const QuantArgs a) {
    using E = Elements<DTYPE>;
    constexpr int kUnroll = 4;
    const uint64_t blocks = static_cast<uint64_t>(a.R) * a.kblocks;
    const uint64_t groups = static_cast<uint64_t>(gridDim.x) * kQuantThreads / E::LANES;
    const uint64_t first = (static_cast<uint64_t>(blockIdx.x) * kQuantThreads + threadIdx.x) / E::LANES;
    const int part = threadIdx.x % E::LANES;
    // whole warps take every trip, so that the shuffles see all of their lanes
    for (uint64_t base = 0; base < blocks; base += kUnroll * groups) {
        E e[kUnroll];
        uint64_t row[kUnroll];
        uint32_t kb[kUnroll];
        bool real[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const uint64_t b = base + first + u * groups;
            real[u] = b < blocks;
            row[u] = real[u] ? b / a.kblocks : 0;
            kb[u] = real[u] ? static_cast<uint32_t>(b - row[u] * a.kblocks) : 0;
            e[u].w = make_uint4(0u, 0u, 0u, 0u);
            if (real[u])
                e[u].template load<VECTOR>(a, static_cast<int64_t>(row[u]), static_cast<int64_t>(kb[u]) * kBlock + part * E::VEC);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            uint32_t m = e[u].largest();
#pragma unroll
            for (int d = E::LANES / 2; d > 0; d >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
            if (!real[u]) continue;
            const float s = scale_of(m);
            const Divisor d(s);
            const int64_t r = static_cast<int64_t>(row[u]);
            const int64_t col = static_cast<int64_t>(kb[u]) * kBlock + part * E::VEC;
            if (d.plain) e[u].template store<VECTOR, true>(a, r, col, d);
            else e[u].template store<VECTOR, false>(a, r, col, d);
            if (part == 0) store_scale(a, r, kb[u], s, 1);
        }
    }
}

// Blocks of 128 rows: one CTA per block, 64 elements per thread.
template <int DTYPE, bool VECTOR>
__global__ void __launch_bounds__(kQuantThreads) quantize_tiles_kernel(const QuantArgs a) {
    using E = Elements<DTYPE>;
    constexpr int kRowsAtOnce = kQuantThreads / E::LANES;
    constexpr int kSteps = kBlock / kRowsAtOnce;
    __shared__ uint32_t most[kQuantThreads / 32];
    const int64_t rb = blockIdx.x / a.kblocks;
    const uint32_t kb = blockIdx.x % a.kblocks;
    const int64_t row0 = rb * kBlock + threadIdx.x / E::LANES;
    const int64_t col = static_cast<int64_t>(kb) * kBlock + threadIdx.x % E::LANES * E::VEC;
    E e[kSteps];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int64_t row = row0 + i * kRowsAtOnce;
        e[i].w = make_uint4(0u, 0u, 0u, 0u);
        if (row < a.R) e[i].template load<VECTOR>(a, row, col);
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) m = max(m, e[i].largest());
    m = __reduce_max_sync(0xffffffffu, m);
    if (threadIdx.x % 32 == 0) most[threadIdx.x / 32] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kQuantThreads / 32; ++i) m = max(m, most[i]);
    const float s = scale_of(m);
    const Divisor d(s);
    const auto store = [&](auto plain) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int64_t row = row0 + i * kRowsAtOnce;
            if (row < a.R) e[i].template store<VECTOR, decltype(plain)::value>(a, row, col, d);
        }
    };
    if (d.plain) store(std::true_type{});
    else store(std::false_type{});
    if (threadIdx.x == 0) store_scale(a, rb, kb, s, kBlock);
}

template <int DTYPE, bool VECTOR>
int launch_quantize(const QuantArgs &a, int64_t block_rows, cudaStream_t stream) {
    if (block_rows == 1) {
        DeviceInfo di;
        if (int rc = current_device_info(&di)) return rc;
        const int64_t per_cta = kQuantThreads / Elements<DTYPE>::LANES;
        const int64_t want = (a.R * a.kblocks + per_cta - 1) / per_cta, most = static_cast<int64_t>(di.sm_count) * 8;
        quantize_rows_kernel<DTYPE, VECTOR><<<static_cast<unsigned>(want < most ? want : most), kQuantThreads, 0, stream>>>(a);
    } else {
        const int64_t tiles = (a.R + kBlock - 1) / kBlock * a.kblocks;
        quantize_tiles_kernel<DTYPE, VECTOR><<<static_cast<unsigned>(tiles), kQuantThreads, 0, stream>>>(a);
    }
    SBW_CUDA_TRY(cudaGetLastError());
    return SBW_OK;
}

}  // namespace
}  // namespace sbw

extern "C" int sbw_quantize_fp8(const void *x, int dtype, int64_t R, int64_t K, int64_t ld, int64_t block_rows, void *out,
                                int64_t ld_out, float *scales, int64_t ld_scales, void *stream) {
    using namespace sbw;
    if (dtype != SBW_DTYPE_F32 && dtype != SBW_DTYPE_BF16) return SBW_ERR_INVALID_ARG;
    if (block_rows != 1 && block_rows != kBlock) return SBW_ERR_INVALID_ARG;
    if (R < 0 || K <= 0 || ld < K || ld_out < K) return SBW_ERR_INVALID_ARG;
    if (K > 0x7fffffffLL - kBlock || R > (int64_t(1) << 40)) return SBW_ERR_UNSUPPORTED;
    const int64_t kblocks = (K + kBlock - 1) / kBlock;
    if (ld_scales < kblocks) return SBW_ERR_INVALID_ARG;
    if (R == 0) return SBW_OK;
    if (!x || !out || !scales) return SBW_ERR_INVALID_ARG;
    const int esize = dtype == SBW_DTYPE_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(x) % esize != 0 || reinterpret_cast<uintptr_t>(scales) % 4 != 0) return SBW_ERR_INVALID_ARG;
    if (block_rows != 1 && (R + kBlock - 1) / kBlock > 0x7fffffffLL / kblocks) return SBW_ERR_UNSUPPORTED;   // the grid
    QuantArgs a;
    a.x = x;
    a.R = R; a.K = K; a.ld = ld;
    a.out = static_cast<uint8_t *>(out);
    a.ld_out = ld_out;
    a.scales = scales;
    a.ld_scales = ld_scales;
    a.kblocks = static_cast<uint32_t>(kblocks);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // 16-byte loads and 8- (bf16) or 4-byte (fp32) stores need rows that start on those boundaries
    const bool vector = reinterpret_cast<uintptr_t>(x) % 16 == 0 && ld * esize % 16 == 0 &&
                        reinterpret_cast<uintptr_t>(out) % (16 / esize) == 0 && ld_out % (16 / esize) == 0;
    if (dtype == SBW_DTYPE_F32)
        return vector ? launch_quantize<SBW_DTYPE_F32, true>(a, block_rows, s) : launch_quantize<SBW_DTYPE_F32, false>(a, block_rows, s);
    return vector ? launch_quantize<SBW_DTYPE_BF16, true>(a, block_rows, s) : launch_quantize<SBW_DTYPE_BF16, false>(a, block_rows, s);
}
