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
            // z Phi(z) = max(z, 0) - |z| erfc(|z| / sqrt(2)) / 2, and
            // erfc(v) = (a1 t + ... + a5 t^5) exp(-v^2) with t = 1 / (1 + 0.3275911 v),
            // off by at most 1.5e-7 (Abramowitz and Stegun, Handbook of Mathematical
            // Functions, 7.1.26); 8192 x 1152 -> 4608 took 139 us with erff, and 124
            const float v = fminf(fabsf(x), 20.f);   // beyond, exp(-v^2 / 2) is 0
            const float t = __builtin_amdgcn_rcpf(fmaf(0.23164189f, v, 1.f));
            float q = fmaf(t, 0.5307027145f, -0.7265760135f);
            q = t * fmaf(t, fmaf(t, fmaf(t, q, 0.7107068705f), -0.142248368f), 0.127414796f);
            z[e] = (x < 0.f ? 0.f : x) - v * (q * __builtin_amdgcn_exp2f(-0.72134752f * v * v));
        } else {
            // z / (1 + exp(-u)): (1 + tanh(u / 2)) / 2 = 1 / (1 + exp(-u)) with
            // u = sqrt(8 / pi) (z + 0.044715 z^3); the exponential in base 2, and
            // v_rcp_f32, within one unit of the last place, for a division's ten
            // instructions
            const float u = act == DFA_ACT_SILU ? -1.4426950408889634f * x : x * fmaf(-0.10294324f, x * x, -2.3022082f);
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
