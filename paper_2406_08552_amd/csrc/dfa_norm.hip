// Layer norm over the features of a token and its gradients, for gfx950 (CDNA4).
//
//   Y  = xh (w + o) + b,  xh = (x - mean) rstd,  rstd = (mean((x - mean)^2) + eps)^(-1/2)
//   dX = rstd (g - mean(g) - xh mean(g xh)),  g = dY (w + o)
//   dw = sum over tokens of dY xh,  db = sum over tokens of dY
//
// Both are HBM streams: a row is read once into registers, where the mean, the
// sum of squared differences (two passes, so that a large mean costs nothing)
// and the result are formed in fp32, and leaves once.  Up to 2048 features a
// wavefront holds a row, 32 values a lane at most; beyond, a workgroup of
// eight wavefronts.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dfa_internal.h"

namespace dfa {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct f32_t {};    // element types of X: fp32,
struct bf16_t {};   // or bf16
template <class T>
struct Bytes;
template <>
struct Bytes<f32_t> {
    static constexpr int N = 4;
};
template <>
struct Bytes<bf16_t> {
    static constexpr int N = 2;
};

// V consecutive elements at p as fp32.  The loads assume the alignment of an
// element only (the hardware takes global accesses at any), so that rows of any
// width are read by vectors; n < V reads the first n and leaves 0 behind them.
template <class T, int V>
__device__ __forceinline__ void load(float (&x)[V], const char* p, int n) {
    if (n >= V) {
        if constexpr (Bytes<T>::N == 4) {
            __builtin_memcpy(x, p, 4 * V);
        } else if constexpr (V == 1) {
            x[0] = __builtin_bit_cast(float, (uint32_t) * (const uint16_t*)p << 16);
        } else {
            uint32_t u[V / 2];
            __builtin_memcpy(u, p, 2 * V);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                x[2 * i] = __builtin_bit_cast(float, u[i] << 16);
                x[2 * i + 1] = __builtin_bit_cast(float, u[i] & 0xFFFF0000u);
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        x[i] = 0.f;
        if (i < n) {
            if constexpr (Bytes<T>::N == 4) x[i] = *(const float*)(p + 4 * i);
            else x[i] = __builtin_bit_cast(float, (uint32_t) * (const uint16_t*)(p + 2 * i) << 16);
        }
    }
}

template <class T, int V>
__device__ __forceinline__ void store(const float (&x)[V], char* p, int n) {
    if constexpr (Bytes<T>::N == 4) {
        if (n >= V) {
            __builtin_memcpy(p, x, 4 * V);
            return;
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) *(float*)(p + 4 * i) = x[i];
    } else {
        if (n >= V && V > 1) {
            uint32_t u[V / 2 > 0 ? V / 2 : 1];
#pragma unroll
            for (int i = 0; i < V / 2; ++i) u[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
            __builtin_memcpy(p, u, 2 * V);
            return;
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) *(uint16_t*)(p + 2 * i) = __builtin_bit_cast(uint16_t, (__bf16)x[i]);
    }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) v += __shfl_xor(v, off);
    return v;
}

// Sum over the WAVES wavefronts that hold a row; `part` is LDS of 2 * WAVES
// values, whose halves alternate so that one barrier per sum is enough.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float* part, int& half) {
    v = wave_sum(v);
    if constexpr (WAVES > 1) {
        float* p = part + half * WAVES;
        half ^= 1;
        if ((threadIdx.x & 63) == 0) p[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v += p[i];
    }
    return v;
}

// How a row lies in registers: WAVES wavefronts, NV vectors of V elements per
// lane; vector k of thread t of the row holds elements V (t + k T) onwards.
template <int V_, int NV_, int WAVES_>
struct Shape {
    static constexpr int V = V_, NV = NV_, WAVES = WAVES_;
    static constexpr int T = 64 * WAVES;                    // threads per row
    static constexpr int ROWS = WAVES == 1 ? 4 : 1;         // rows of a workgroup at a time
    static constexpr int NT = T * ROWS;
    static constexpr int C_MAX = V * NV * T;
};

struct NormParams {
    const char* X;
    const char* dY;
    Rows weight, bias;
    float offset, eps;
    char* out;               // Y, or dX
    float* mean;
    float* rstd;
    float* partial;          // backward: [groups][splits][2][C], or null
    float* dweight;          // backward, splits = 1: the sums themselves (each may be null)
    float* dbias;
    int M, L, C;
    int rows;                // rows per wavefront (or workgroup) and
    int group_rows, splits;  // backward: tokens of a group, workgroups that share them
};

// Rows [first, last) of one wavefront or workgroup, weights kept while the batch entry stays.
template <class XT, class S>
__global__ void __launch_bounds__(S::NT) norm_kernel(NormParams p) {
    __shared__ float part[2 * S::WAVES];
    constexpr int V = S::V, NV = S::NV;
    const int t = S::WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int unit = S::WAVES == 1 ? blockIdx.x * S::ROWS + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x;
    const long long first = (long long)unit * p.rows;
    const int last = (int)min((long long)p.M, first + p.rows);
    const float inv = 1.f / (float)p.C;
    int half = 0, entry = -1;
    float w[NV][V], b[NV][V];
    for (int row = (int)min(first, (long long)p.M); row < last; ++row) {
        const char* x0 = p.X + (size_t)row * p.C * Bytes<XT>::N;
        float x[NV][V];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = V * (t + k * S::T);
            load<XT, V>(x[k], x0 + (size_t)c * Bytes<XT>::N, p.C - c);
        }
        const int e = row / p.L;
        if (e != entry) {
            entry = e;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = V * (t + k * S::T);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    w[k][i] = 1.f;
                    b[k][i] = 0.f;
                }
                if (p.weight.p) {
                    load<f32_t, V>(w[k], (const char*)(p.weight.p + (size_t)e * p.weight.stride + c), p.C - c);
#pragma unroll
                    for (int i = 0; i < V; ++i) w[k][i] += p.offset;
                }
                if (p.bias.p) load<f32_t, V>(b[k], (const char*)(p.bias.p + (size_t)e * p.bias.stride + c), p.C - c);
            }
        }
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) s += x[k][i];
        const float mean = row_sum<S::WAVES>(s, part, half) * inv;
        s = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[k][i] -= mean;
                const bool in = V * (t + k * S::T) + i < p.C;
                s += in ? x[k][i] * x[k][i] : 0.f;
            }
        const float rstd = 1.f / sqrtf(row_sum<S::WAVES>(s, part, half) * inv + p.eps);
        if (t == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
        char* y0 = p.out + (size_t)row * p.C * 2;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = V * (t + k * S::T);
#pragma unroll
            for (int i = 0; i < V; ++i) x[k][i] = x[k][i] * rstd * w[k][i] + b[k][i];
            store<bf16_t, V>(x[k], y0 + (size_t)c * 2, p.C - c);
        }
    }
}

// dX of the workgroup's rows, and its share of dweight and dbias: every lane
// sums its own columns over the rows of its wavefront, then the wavefronts of
// the workgroup are added in LDS.
template <class XT, class S>
__global__ void __launch_bounds__(S::NT) norm_grad_kernel(NormParams p) {
    __shared__ float part[2 * S::WAVES];
    __shared__ float cols[S::ROWS > 1 ? S::C_MAX : 1];
    constexpr int V = S::V, NV = S::NV;
    const int t = S::WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int wave = S::WAVES == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const int group = blockIdx.x / p.splits, split = blockIdx.x % p.splits;
    const int rows = p.rows * S::ROWS;   // of the workgroup
    const long long base = (long long)group * p.group_rows;
    const long long end = base + min((long long)p.group_rows, (long long)(split + 1) * rows);
    const long long first = min(end, base + (long long)split * rows + (long long)wave * p.rows);
    const long long last = min(end, first + p.rows);
    const float inv = 1.f / (float)p.C;
    int half = 0, entry = -1;
    float w[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) dw[k][i] = db[k][i] = 0.f;
    for (int row = (int)first; row < (int)last; ++row) {
        float x[NV][V], g[NV][V];
        const char* x0 = p.X + (size_t)row * p.C * Bytes<XT>::N;
        const char* g0 = p.dY + (size_t)row * p.C * 2;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = V * (t + k * S::T);
            load<XT, V>(x[k], x0 + (size_t)c * Bytes<XT>::N, p.C - c);
            load<bf16_t, V>(g[k], g0 + (size_t)c * 2, p.C - c);
        }
        const int e = row / p.L;
        if (e != entry) {
            entry = e;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = V * (t + k * S::T);
#pragma unroll
                for (int i = 0; i < V; ++i) w[k][i] = 1.f;
                if (p.weight.p) {
                    load<f32_t, V>(w[k], (const char*)(p.weight.p + (size_t)e * p.weight.stride + c), p.C - c);
#pragma unroll
                    for (int i = 0; i < V; ++i) w[k][i] += p.offset;
                }
            }
        }
        const float mean = p.mean[row], rstd = p.rstd[row];
        float sg = 0.f, sx = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = (x[k][i] - mean) * rstd;
                db[k][i] += g[k][i];
                dw[k][i] += g[k][i] * xh;
                g[k][i] *= w[k][i];
                x[k][i] = xh;
                const bool in = V * (t + k * S::T) + i < p.C;   // g is 0 behind the row, xh is not
                sg += g[k][i];
                sx += in ? g[k][i] * xh : 0.f;
            }
        sg = row_sum<S::WAVES>(sg, part, half) * inv;
        sx = row_sum<S::WAVES>(sx, part, half) * inv;
        char* d0 = p.out + (size_t)row * p.C * Bytes<XT>::N;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = V * (t + k * S::T);
#pragma unroll
            for (int i = 0; i < V; ++i) x[k][i] = rstd * (g[k][i] - sg - x[k][i] * sx);
            store<XT, V>(x[k], d0 + (size_t)c * Bytes<XT>::N, p.C - c);
        }
    }
    if (!p.partial && !p.dweight && !p.dbias) return;
    float* to[2] = {p.dweight ? p.dweight + (size_t)group * p.C : nullptr, p.dbias ? p.dbias + (size_t)group * p.C : nullptr};
    if (p.partial) {
        to[0] = p.partial + (size_t)blockIdx.x * 2 * p.C;
        to[1] = to[0] + p.C;
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float(&d)[NV][V] = which ? db : dw;
        if constexpr (S::ROWS > 1) {
            for (int r = 1; r < S::ROWS; ++r) {   // in the order of the wavefronts
                __syncthreads();
                if (wave == r) {
#pragma unroll
                    for (int k = 0; k < NV; ++k)
#pragma unroll
                        for (int i = 0; i < V; ++i) cols[(k * V + i) * 64 + t] = d[k][i];
                }
                __syncthreads();
                if (wave == 0) {
#pragma unroll
                    for (int k = 0; k < NV; ++k)
#pragma unroll
                        for (int i = 0; i < V; ++i) d[k][i] += cols[(k * V + i) * 64 + t];
                }
            }
        }
        if (wave == 0 && to[which]) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = V * (t + k * S::T);
                store<f32_t, V>(d[k], (char*)(to[which] + c), p.C - c);
            }
        }
    }
}

// dweight and dbias of a group: the sums of its splits' partial sums.  16
// wavefronts read every 16th split of 64 columns, then are added in order.
__global__ void __launch_bounds__(1024) norm_sum_kernel(const float* partial, float* dweight, float* dbias, int C, int splits) {
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = blockIdx.x * 64 + lane;      // of 2 C
    const float* from = partial + (size_t)blockIdx.y * splits * 2 * C + col;
    float v = 0.f;
    if (col < 2 * C)
        for (int i = wave; i < splits; i += 16) v += from[(size_t)i * 2 * C];
    s[wave][lane] = v;
    __syncthreads();
    if (wave || col >= 2 * C) return;
    for (int i = 1; i < 16; ++i) v += s[i][lane];
    float* to = col < C ? dweight : dbias;
    if (to) to[(size_t)blockIdx.y * C + (col < C ? col : col - C)] = v;
}

// Tokens per wavefront (or workgroup, above 2048 features) and splits of a
// group's tokens in the backward pass.
struct Split {
    int rows, splits, per_block;
};
Split grad_split(int B, int L, int C, int groups) {
    const long long M = (long long)B * L, group_rows = M / groups;
    const int block = C <= 2048 ? 4 : 1;
    // about 512 workgroups, each of 4 rows per wavefront at least
    long long splits = (512 + groups - 1) / groups;
    long long rows = (group_rows + splits * block - 1) / (splits * block);
    if (rows < 4) rows = 4;
    splits = (group_rows + rows * block - 1) / (rows * block);
    return Split{(int)rows, (int)splits, block};
}

template <class XT, class S>
hipError_t run_norm(NormParams& p, hipStream_t stream) {
    const long long units = 256LL * 16 / S::WAVES;
    p.rows = (int)((p.M + units - 1) / units);
    const long long per_block = (long long)p.rows * S::ROWS;
    const int blocks = (int)((p.M + per_block - 1) / per_block);
    hipLaunchKernelGGL((norm_kernel<XT, S>), dim3(blocks), dim3(S::NT), 0, stream, p);
    return hipGetLastError();
}

template <class XT, class S>
hipError_t run_grad(NormParams& p, int groups, hipStream_t stream) {
    hipLaunchKernelGGL((norm_grad_kernel<XT, S>), dim3((unsigned)(groups * p.splits)), dim3(S::NT), 0, stream, p);
    return hipGetLastError();
}

template <class XT, class F>
hipError_t by_width(int C, F&& run) {
    if (C <= 512) return run(Shape<4, 2, 1>{});
    if (C <= 1280) return run(Shape<4, 5, 1>{});
    if (C <= 2048) return run(Shape<4, 8, 1>{});
    if (C <= 4096) return run(Shape<4, 2, 8>{});
    return run(Shape<4, 8, 8>{});
}

}  // namespace

size_t norm_grad_partials(int B, int L, int C, int groups) {
    const Split s = grad_split(B, L, C, groups);
    return s.splits > 1 ? (size_t)groups * s.splits * 2 * C : 0;
}

hipError_t launch_layer_norm(const NormLaunch& a, hipStream_t stream) {
    NormParams p{};
    p.X = (const char*)a.X;
    p.weight = a.weight;
    p.bias = a.bias;
    p.offset = a.offset;
    p.eps = a.eps;
    p.out = (char*)a.Y;
    p.mean = a.mean;
    p.rstd = a.rstd;
    p.M = a.B * a.L;
    p.L = a.L;
    p.C = a.C;
    if (a.x_f32) return by_width<f32_t>(a.C, [&](auto s) { return run_norm<f32_t, decltype(s)>(p, stream); });
    return by_width<bf16_t>(a.C, [&](auto s) { return run_norm<bf16_t, decltype(s)>(p, stream); });
}

hipError_t launch_layer_norm_backward(const NormGradLaunch& a, hipStream_t stream) {
    const Split split = grad_split(a.B, a.L, a.C, a.groups);
    const bool sums = a.dweight || a.dbias;
    NormParams p{};
    p.X = (const char*)a.X;
    p.dY = (const char*)a.dY;
    p.weight = a.weight;
    p.offset = a.offset;
    p.out = (char*)a.dX;
    p.mean = (float*)a.mean;
    p.rstd = (float*)a.rstd;
    p.M = a.B * a.L;
    p.L = a.L;
    p.C = a.C;
    p.group_rows = p.M / a.groups;
    p.rows = split.rows;
    p.splits = split.splits;
    const bool two = sums && split.splits > 1;
    if (two) p.partial = a.partial;
    else {
        p.dweight = a.dweight;
        p.dbias = a.dbias;
    }
    const hipError_t e =
        a.x_f32 ? by_width<f32_t>(a.C, [&](auto s) { return run_grad<f32_t, decltype(s)>(p, a.groups, stream); })
                : by_width<bf16_t>(a.C, [&](auto s) { return run_grad<bf16_t, decltype(s)>(p, a.groups, stream); });
    if (e != hipSuccess || !two) return e;
    hipLaunchKernelGGL(norm_sum_kernel, dim3((2 * a.C + 63) / 64, a.groups), dim3(1024), 0, stream, a.partial, a.dweight,
                       a.dbias, a.C, split.splits);
    return hipGetLastError();
}

}  // namespace dfa
