// Linear layer for gfx950 (CDNA4): Y = residual + gate * act(X W^T + bias),
// fp32 from the accumulators to the one rounding of Y.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dfa_epilogue.h"
#include "dfa_internal.h"

namespace dfa {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct LinearParams {
    const uint16_t* X;
    const uint16_t* W;
    const float* bias;
    Rows gate;
    const void* residual;
    void* Y;
    int act;
    int M, N, K, L, H, d;      // d = K / H
    int nft, ntt;              // feature and token tiles
};

// Eight consecutive k of a row at p, of which n are there (n >= 8: all), zeros behind.
__device__ __forceinline__ u32x4 load8(const uint16_t* p, int n) {
    u32x4 v{0, 0, 0, 0};
    if (n >= 8) {
        __builtin_memcpy(&v, p, 16);
    } else {
        uint16_t e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i < n ? p[i] : (uint16_t)0;
        __builtin_memcpy(&v, e, 16);
    }
    return v;
}

// 64 features x 64 tokens per workgroup of four wavefronts, k by 32.
template <bool YF32>
__global__ void __launch_bounds__(256) linear_general_kernel(LinearParams p) {
    constexpr int PITCH = 40;   // elements of an LDS row
    __shared__ __attribute__((aligned(16))) uint16_t sx[64 * PITCH], sw[64 * PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r32 = lane & 31, h = lane >> 5;
    const int t0 = (blockIdx.x / p.nft) * 64, n0 = (blockIdx.x % p.nft) * 64;
    const int row = tid >> 2, ch = (tid & 3) * 8;
    const int t = min(t0 + row, p.M - 1);
    const uint16_t* xr = p.X;
    const int b = t / p.L;
    if (p.H == 1) xr += (size_t)t * p.K;
    else xr += ((size_t)b * p.H * p.L + (t - b * p.L)) * p.d;
    const uint16_t* wr = p.W + (size_t)min(n0 + row, p.N - 1) * p.K;
    const int wt = wave & 1, wf = wave >> 1;
    const int f = n0 + 32 * wf + r32;
    const float bias = p.bias ? p.bias[min(f, p.N - 1)] : 0.f;
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = bias;
    for (int k0 = 0; k0 < p.K; k0 += 32) {
        const int k = k0 + ch;
        u32x4 xv{0, 0, 0, 0}, wv{0, 0, 0, 0};
        if (k < p.K) {
            // heads: a chunk of eight lies in one head (d % 8 = 0)
            const uint16_t* at = p.H == 1 ? xr + k : xr + (size_t)(k / p.d) * p.L * p.d + k % p.d;
            xv = load8(at, p.K - k);
            wv = load8(wr + k, p.K - k);
        }
        __syncthreads();
        *(u32x4*)(sx + row * PITCH + ch) = xv;
        *(u32x4*)(sw + row * PITCH + ch) = wv;
        __syncthreads();
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const bf16x8 a = __builtin_bit_cast(bf16x8, *(const u32x4*)(sx + (32 * wt + r32) * PITCH + 16 * ks + 8 * h));
            const bf16x8 w = __builtin_bit_cast(bf16x8, *(const u32x4*)(sw + (32 * wf + r32) * PITCH + 16 * ks + 8 * h));
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, w, acc, 0, 0, 0);
        }
    }
    if (f >= p.N) return;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int tt = t0 + 32 * wt + 8 * (i / 4) + 4 * h + i % 4;
        if (tt >= p.M) continue;
        float z[1] = {acc[i]}, r[1] = {0.f};
        const size_t o = ((size_t)tt * p.N + f) * (YF32 ? 4 : 2);
        if (p.residual) read_row<YF32, 1>(r, (const char*)p.residual + o);
        activate<1>(z, p.act);
        z[0] = fmaf(z[0], p.gate.p ? p.gate.p[(size_t)(tt / p.L) * p.gate.stride + f] : 1.f, r[0]);
        write_row<YF32, 1>(z, (char*)p.Y + o);
    }
}

}  // namespace

hipError_t launch_linear(const LinearLaunch& a, hipStream_t stream) {
    if (a.K % (a.H > 1 ? 128 : 8) == 0) return launch_linear_tiles(a, stream);
    LinearParams p{};
    p.X = (const uint16_t*)a.X;
    p.W = (const uint16_t*)a.W;
    p.bias = a.bias;
    p.gate = a.gate;
    p.residual = a.residual;
    p.Y = a.Y;
    p.act = a.act;
    p.M = a.B * a.L;
    p.N = a.N;
    p.K = a.K;
    p.L = a.L;
    p.H = a.H;
    p.d = a.K / a.H;
    p.nft = (p.N + 63) / 64;
    p.ntt = (p.M + 63) / 64;
    const long long blocks = (long long)p.nft * p.ntt;
    if (blocks > (1LL << 23)) return hipErrorInvalidValue;
    if (a.y_f32) hipLaunchKernelGGL(linear_general_kernel<true>, dim3((unsigned)blocks), dim3(256), 0, stream, p);
    else hipLaunchKernelGGL(linear_general_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace dfa
