// What the linear layer's kernels do with an accumulated value, in one place so
// that all give the same bits: y = residual + gate * act(z), fp32 until the
// one rounding of y.
#ifndef DFA_EPILOGUE_H
#define DFA_EPILOGUE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dfa.h"

namespace dfa {

template <int E>
__device__ __forceinline__ void activate(float (&z)[E], int act) {
    if (act == DFA_ACT_NONE) return;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float x = z[e];
        if (act == DFA_ACT_GELU) {
            const float half = 0.5f * x;
            z[e] = fmaf(half, erff(x * 0.70710678118654752f), half);
        } else {
            // (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u)), u = sqrt(2 / pi) (x + 0.044715 x^3)
            // the exponential in base 2; v_rcp_f32 is within one unit of the last place, where a division takes ten instructions
            const float u = act == DFA_ACT_SILU ? -1.4426950408889634f * x
                                                : x * fmaf(-0.10294324f, x * x, -2.3022082f);
            z[e] = x * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(u));
        }
    }
}

// E neighbouring values of a row of Y or of the residual, at the alignment of
// one element (rows of any width; the hardware takes global accesses at any).
template <bool F32, int E>
__device__ __forceinline__ void read_row(float (&x)[E], const char* p) {
    if constexpr (F32) {
        __builtin_memcpy(x, p, 4 * E);
    } else if constexpr (E % 2 == 0) {
        uint32_t u[E / 2];
        __builtin_memcpy(u, p, 2 * E);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            x[2 * i] = __builtin_bit_cast(float, u[i] << 16);
            x[2 * i + 1] = __builtin_bit_cast(float, u[i] & 0xFFFF0000u);
        }
    } else {
        static_assert(E == 1, "one, or an even number");
        x[0] = __builtin_bit_cast(float, (uint32_t) * (const uint16_t*)p << 16);
    }
}
template <bool F32, int E>
__device__ __forceinline__ void write_row(const float (&x)[E], char* p) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    if constexpr (F32) {
        __builtin_memcpy(p, x, 4 * E);
    } else if constexpr (E % 2 == 0) {
        uint32_t u[E / 2];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) u[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
        __builtin_memcpy(p, u, 2 * E);
    } else {
        static_assert(E == 1, "one, or an even number");
        *(uint16_t*)p = __builtin_bit_cast(uint16_t, (__bf16)x[0]);
    }
}

}  // namespace dfa

#endif
