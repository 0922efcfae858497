// What the kernels that look at watermarked logits share: a row's seed, the green test of its
// columns, and Eq. 2 on one logit or on a packed pair.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "../../include/sbw.h"
#include "sbw_hash.cuh"

namespace sbw {

__device__ __forceinline__ uint32_t add_bf16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// 2^x to 2 ulp with results below 2^-126 flushed to zero (one instruction instead of a scaled
// sequence): for terms of a sum whose largest term is 1.
__device__ __forceinline__ float ex2_approx_ftz(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <int SCHEME>
struct RowSeedS;
template <>
struct RowSeedS<SBW_SCHEME_CONTEXT> {
    RowKeys rk;
    __device__ __forceinline__ void init(uint64_t key, const int32_t *ctx, int W) {
        rk = make_row_keys(seed_context(key, ctx, W));
    }
    __device__ __forceinline__ uint32_t word0(uint32_t v, uint64_t, const Weyl) const {
        return philox_word0(v, rk);
    }
    template <int N>
    __device__ __forceinline__ void word0_n(uint32_t vg, uint64_t, const Weyl, uint32_t (&x)[N]) const {
        philox_word0_n<N>(vg, rk, x);
    }
};
template <>
struct RowSeedS<SBW_SCHEME_SELFSALT> {
    uint32_t jmin;
    __device__ __forceinline__ void init(uint64_t, const int32_t *ctx, int W) { jmin = jenkins_min(ctx, W); }
    __device__ __forceinline__ uint32_t word0(uint32_t v, uint64_t key, const Weyl w) const {
        return philox_word0(v, seed_selfsalt(key, jmin, v), w);
    }
    template <int N>
    __device__ __forceinline__ void word0_n(uint32_t vg, uint64_t key, const Weyl w, uint32_t (&x)[N]) const {
        uint32_t v[N];
        uint64_t r[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = vg + i;
            r[i] = seed_selfsalt(key, jmin, v[i]);
        }
        philox_word0_n<N>(v, r, x, w);
    }
};

// A row whose logits are taken as they are.
constexpr int kSchemeNone = -1;
template <>
struct RowSeedS<kSchemeNone> {
    __device__ __forceinline__ void init(uint64_t, const int32_t *, int) {}
};

// Biased logit of one element, widened to fp32 (Eq. 2 in the logits' own precision).
template <int DTYPE>
__device__ __forceinline__ float biased(uint32_t raw, bool green, float delta) {
    if constexpr (DTYPE == SBW_DTYPE_F32) {
        const float x = __uint_as_float(raw);
        return green ? __fadd_rn(x, delta) : x;
    } else {
        const float x = __uint_as_float(raw << 16);
        // fp32 sum of two bf16 values, rounded once more to bf16 = correctly rounded bf16 sum
        return green ? __bfloat162float(__float2bfloat16_rn(__fadd_rn(x, delta))) : x;
    }
}

// What Eq. 1 and Eq. 2 need apart from the row's seed.
struct BiasParams {
    uint64_t key;
    uint32_t thr_m1;
    float delta;           // in the logits' precision, widened
    uint32_t delta_bf16;   // bf16 bits of delta
    Weyl weyl;
};

// Eq. 1 + Eq. 2 on the 4 (fp32) or 8 (bf16) logits of a vector; vg is the first one's global id.
template <int DTYPE, int SCHEME>
__device__ __forceinline__ void bias_vector(uint4 &w, const RowSeedS<SCHEME> &rs, uint32_t vg, const BiasParams &p) {
    if constexpr (SCHEME != kSchemeNone) {
        constexpr int VEC = DTYPE == SBW_DTYPE_F32 ? 4 : 8;
        uint32_t x[VEC];
        rs.template word0_n<VEC>(vg, p.key, p.weyl, x);
        uint32_t *e = reinterpret_cast<uint32_t *>(&w);
        if constexpr (DTYPE == SBW_DTYPE_F32) {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (x[i] <= p.thr_m1) e[i] = __float_as_uint(__fadd_rn(__uint_as_float(e[i]), p.delta));
        } else {
            // one packed bf16 add per pair with {delta or -0.0} per half
            const uint32_t dlo = p.delta_bf16, dhi = p.delta_bf16 << 16;
#pragma unroll
            for (int i = 0; i < VEC / 2; ++i) {
                const uint32_t d = (x[2 * i] <= p.thr_m1 ? dlo : 0x8000u) | (x[2 * i + 1] <= p.thr_m1 ? dhi : 0x80000000u);
                e[i] = add_bf16x2(e[i], d);
            }
        }
    }
}

// The same on one logit in memory: column `col` of a row, widened.
template <int DTYPE, int SCHEME>
__device__ __forceinline__ float biased_at(const char *row_ptr, uint32_t col, const RowSeedS<SCHEME> &rs, uint32_t vg,
                                           const BiasParams &p) {
    uint32_t raw;
    if constexpr (DTYPE == SBW_DTYPE_F32) raw = reinterpret_cast<const uint32_t *>(row_ptr)[col];
    else raw = reinterpret_cast<const uint16_t *>(row_ptr)[col];
    if constexpr (SCHEME == kSchemeNone) return __uint_as_float(DTYPE == SBW_DTYPE_F32 ? raw : raw << 16);
    else return biased<DTYPE>(raw, rs.word0(vg, p.key, p.weyl) <= p.thr_m1, p.delta);
}

}  // namespace sbw
