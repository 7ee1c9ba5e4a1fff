// Layer norm over the features of a token and its gradients, for gfx950 (CDNA4).
//
//   Y  = xh (w + o) + b,  xh = (x - mean) rstd,  rstd = (mean((x - mean)^2) + eps)^(-1/2)
//   dX = rstd (g - mean(g) - xh mean(g xh)),  g = dY (w + o)
//   dw = sum over tokens of dY xh,  db = sum over tokens of dY
//
// Both are HBM streams: a row is read once into registers, where the mean, the
// sum of squared differences (two passes, so that a large mean costs nothing)
// and the result are formed in fp32, and leaves once.  Up to 1280 features a
// wavefront holds a row, 20 values a lane at most; beyond, a workgroup of
// four or sixteen wavefronts (1152 features by four: 32768 tokens 54 us against
// 49, gradients of 8192 32 against 19; 4096 features by sixteen: 60 against 44).
// A wavefront walks several rows of a batch entry, whose weights it keeps, and
// reads the next row while it works on this one.
//
// 32768 tokens x 1152 fp32 to bf16 take 49 us, 4.6 TB/s where a large copy
// reaches 5.1; the gradients of 8192 tokens x 1152 bf16 15 us, 3.7 TB/s, of
// which 4 us are the second kernel's, which adds up the workgroups' sums.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dfa_internal.h"

namespace dfa {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    const int x = __builtin_bit_cast(int, v);
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, x, CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float lane_value(float v, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}
// Sum over the wavefront, the same in every lane: within rows of 16 lanes by
// DPP (xor 1, xor 2, mirrored halves, mirrored row), then the four rows.
__device__ __forceinline__ float wave_sum(float v) {
    v = dpp_add<0xB1>(v);
    v = dpp_add<0x4E>(v);
    v = dpp_add<0x141>(v);
    v = dpp_add<0x140>(v);
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
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
// lane.  Vector k of thread t covers the V elements from V (t + k T) on; where
// V does not divide C, the last vector of the row is moved back to end with it
// (so that no access is partial) and covers some elements of its neighbour
// again: both form the same values, and sums leave the second ones out.
template <int V_, int NV_, int WAVES_, int ROWS_, bool EXACT_>
struct Shape {
    static constexpr int V = V_, NV = NV_, WAVES = WAVES_;
    static constexpr bool EXACT = EXACT_;                   // V divides C
    static constexpr int T = 64 * WAVES;                    // threads per row
    static constexpr int ROWS = WAVES == 1 ? ROWS_ : 1;     // rows of a workgroup at a time
    static constexpr int NT = T * ROWS;
    static constexpr bool AHEAD = WAVES <= 4;               // reads the next row early (sixteen wavefronts have no registers left)
    static constexpr int C_MAX = V * NV * T;
};

template <class S>
struct Place {
    int c[S::NV];       // first element
    int again[S::NV];   // how many of its first elements the neighbour has too
    bool in[S::NV];
    __device__ __forceinline__ Place(int t, int C) {
#pragma unroll
        for (int k = 0; k < S::NV; ++k) {
            const int at = S::V * (t + k * S::T);
            in[k] = at < C;
            c[k] = S::EXACT ? at : min(at, C - S::V);
            again[k] = S::EXACT ? 0 : at - c[k];
        }
    }
    __device__ __forceinline__ bool counts(int k, int i) const { return S::EXACT || i >= again[k]; }
};

// One row of fp32 or bf16 values as loaded.  The loads assume the alignment of
// an element only: the hardware takes global accesses at any.
template <class S, bool F32>
struct Raw {
    static constexpr int W = F32 ? S::V : (S::V + 1) / 2;   // registers of a vector
    static constexpr int SZ = F32 ? 4 : 2;
    uint32_t u[S::NV][W];
    __device__ __forceinline__ void load(const void* row, const Place<S>& at) {
#pragma unroll
        for (int k = 0; k < S::NV; ++k) {
#pragma unroll
            for (int i = 0; i < W; ++i) u[k][i] = 0;
            if (at.in[k]) __builtin_memcpy(u[k], (const char*)row + (size_t)at.c[k] * SZ, S::V * SZ);
        }
    }
    __device__ __forceinline__ float get(int k, int i) const {
        if constexpr (F32) return __builtin_bit_cast(float, u[k][i]);
        else return __builtin_bit_cast(float, i & 1 ? u[k][i / 2] & 0xFFFF0000u : u[k][i / 2] << 16);
    }
};

template <class S, bool F32>
__device__ __forceinline__ void store_row(const float (&x)[S::NV][S::V], void* row, const Place<S>& at) {
#pragma unroll
    for (int k = 0; k < S::NV; ++k) {
        if (!at.in[k]) continue;
        char* to = (char*)row + (size_t)at.c[k] * (F32 ? 4 : 2);
        if constexpr (F32) {
            __builtin_memcpy(to, x[k], 4 * S::V);
        } else if constexpr (S::V == 1) {
            *(uint16_t*)to = __builtin_bit_cast(uint16_t, (__bf16)x[k][0]);
        } else {
            uint32_t u[S::V / 2];
#pragma unroll
            for (int i = 0; i < S::V / 2; ++i)
                u[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[k][2 * i], (__bf16)x[k][2 * i + 1]});
            __builtin_memcpy(to, u, 2 * S::V);
        }
    }
}

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

// The batch entry's weights plus the offset (no weights: 1), or its biases (none: 0).
template <class S>
__device__ __forceinline__ void load_vectors(float (&v)[S::NV][S::V], const Rows& r, int entry, float offset, float none,
                                             const Place<S>& at) {
    if (!r.p) {
#pragma unroll
        for (int k = 0; k < S::NV; ++k)
#pragma unroll
            for (int i = 0; i < S::V; ++i) v[k][i] = none;
        return;
    }
    Raw<S, true> raw;
    raw.load(r.p + (size_t)entry * r.stride, at);
#pragma unroll
    for (int k = 0; k < S::NV; ++k)
#pragma unroll
        for (int i = 0; i < S::V; ++i) v[k][i] = raw.get(k, i) + offset;
}

template <bool F32, class S>
__global__ void __launch_bounds__(S::NT) norm_kernel(NormParams p) {
    __shared__ float part[2 * S::WAVES];
    constexpr int V = S::V, NV = S::NV, SZ = F32 ? 4 : 2;
    const int t = S::WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int unit = S::WAVES == 1 ? blockIdx.x * S::ROWS + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x;
    const long long first = (long long)unit * p.rows;
    if (first >= p.M) return;
    const int last = (int)min((long long)p.M, first + p.rows);
    const float inv = 1.f / (float)p.C;
    const Place<S> at(t, p.C);
    int half = 0, entry = -1;
    float w[NV][V], b[NV][V];
    Raw<S, F32> next;
    if constexpr (S::AHEAD) next.load(p.X + (size_t)first * p.C * SZ, at);
    for (int row = (int)first; row < last; ++row) {
        if constexpr (!S::AHEAD) next.load(p.X + (size_t)row * p.C * SZ, at);
        const Raw<S, F32> raw = next;
        if (S::AHEAD && row + 1 < last) next.load(p.X + (size_t)(row + 1) * p.C * SZ, at);
        const int e = row / p.L;
        if (e != entry) {
            entry = e;
            load_vectors<S>(w, p.weight, e, p.offset, 1.f, at);
            load_vectors<S>(b, p.bias, e, 0.f, 0.f, at);
        }
        float x[NV][V], s = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[k][i] = raw.get(k, i);   // 0 behind the row
                s += at.counts(k, i) ? x[k][i] : 0.f;
            }
        const float mean = row_sum<S::WAVES>(s, part, half) * inv;
        s = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[k][i] -= mean;
                const float d = at.in[k] && at.counts(k, i) ? x[k][i] : 0.f;
                s += d * d;
            }
        const float rstd = 1.f / sqrtf(row_sum<S::WAVES>(s, part, half) * inv + p.eps);
        if (t == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) x[k][i] = x[k][i] * rstd * w[k][i] + b[k][i];
        store_row<S, false>(x, p.out + (size_t)row * p.C * 2, at);
    }
}

// dX of the workgroup's rows, and its share of dweight and dbias: every lane
// sums its own columns over the rows of its wavefront, then the wavefronts of
// the workgroup are added in LDS, in order.
template <bool F32, class S>
__global__ void __launch_bounds__(S::NT) norm_grad_kernel(NormParams p) {
    __shared__ float part[2 * S::WAVES];
    constexpr int V = S::V, NV = S::NV, SZ = F32 ? 4 : 2;
    __shared__ __attribute__((aligned(16))) float cols[S::ROWS][S::ROWS > 1 ? S::C_MAX : 4];
    const int t = S::WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int wave = S::WAVES == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const int group = blockIdx.x / p.splits, split = blockIdx.x % p.splits;
    const long long base = (long long)group * p.group_rows, end = base + p.group_rows;
    const long long first = min(end, base + ((long long)split * S::ROWS + wave) * p.rows);
    const int last = (int)min(end, first + p.rows);
    const float inv = 1.f / (float)p.C;
    const Place<S> at(t, p.C);
    int half = 0, entry = -1;
    float w[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) dw[k][i] = db[k][i] = 0.f;
    Raw<S, F32> nx;
    Raw<S, false> ng;
    float nmean = 0.f, nrstd = 0.f;
    auto fetch = [&](int row) {
        nx.load(p.X + (size_t)row * p.C * SZ, at);
        ng.load(p.dY + (size_t)row * p.C * 2, at);
        nmean = p.mean[row];
        nrstd = p.rstd[row];
    };
    if (S::AHEAD && first < last) fetch((int)first);
    for (int row = (int)first; row < last; ++row) {
        if constexpr (!S::AHEAD) fetch(row);
        const Raw<S, F32> rx = nx;
        const Raw<S, false> rg = ng;
        const float mean = nmean, rstd = nrstd;
        if (S::AHEAD && row + 1 < last) fetch(row + 1);
        const int e = row / p.L;
        if (e != entry) {
            entry = e;
            load_vectors<S>(w, p.weight, e, p.offset, 1.f, at);
        }
        float x[NV][V], g[NV][V], sg = 0.f, sx = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = (rx.get(k, i) - mean) * rstd, dy = rg.get(k, i);   // dy is 0 behind the row
                db[k][i] += dy;
                dw[k][i] += dy * xh;
                x[k][i] = xh;
                g[k][i] = dy * w[k][i];
                const float gc = at.counts(k, i) ? g[k][i] : 0.f;
                sg += gc;
                sx += gc * xh;
            }
        sg = row_sum<S::WAVES>(sg, part, half) * inv;
        sx = row_sum<S::WAVES>(sx, part, half) * inv;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) x[k][i] = rstd * (g[k][i] - sg - x[k][i] * sx);
        store_row<S, F32>(x, p.out + (size_t)row * p.C * SZ, at);
    }
    if (!p.partial && !p.dweight && !p.dbias) return;
    float* to[2] = {p.dweight ? p.dweight + (size_t)group * p.C : nullptr, p.dbias ? p.dbias + (size_t)group * p.C : nullptr};
    if (p.partial) {
        to[0] = p.partial + (size_t)blockIdx.x * 2 * p.C;
        to[1] = to[0] + p.C;
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const float(&d)[NV][V] = which ? db : dw;
        if constexpr (S::ROWS > 1) {
            __syncthreads();
            store_row<S, true>(d, cols[wave], at);
            __syncthreads();
            if (to[which])
                for (int c = threadIdx.x; c < p.C; c += S::NT) {
                    float v = 0.f;
#pragma unroll
                    for (int r = 0; r < S::ROWS; ++r) v += cols[r][c];
                    to[which][c] = v;
                }
        } else if (to[which]) {
            store_row<S, true>(d, to[which], at);
        }
    }
}

// dweight and dbias of a group: the sums of its splits' partial sums.  16
// wavefronts read every 16th split of 64 columns, AT of them in flight, then
// are added in order.
template <int AT>
__global__ void __launch_bounds__(1024) norm_sum_kernel(const float* partial, float* dweight, float* dbias, int C, int splits) {
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = blockIdx.x * 64 + lane;      // of 2 C
    const float* from = partial + (size_t)blockIdx.y * splits * 2 * C + col;
    float v = 0.f;
    if (col < 2 * C) {
        for (int i = wave; i < splits; i += 16 * AT) {
            float x[AT];   // behind the end the last one again, which is not added
#pragma unroll
            for (int j = 0; j < AT; ++j) x[j] = from[(size_t)min(i + 16 * j, splits - 1) * 2 * C];
#pragma unroll
            for (int j = 0; j < AT; ++j) v += i + 16 * j < splits ? x[j] : 0.f;
        }
    }
    s[wave][lane] = v;
    __syncthreads();
    if (wave || col >= 2 * C) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) v += s[i][lane];
    float* to = col < C ? dweight : dbias;
    if (to) to[(size_t)blockIdx.y * C + (col < C ? col : col - C)] = v;
}

constexpr int WIDE = 1280;       // features that one wavefront holds
constexpr int GRAD_ROWS = 8;     // wavefronts of a workgroup, backward, and
constexpr int FORWARD_ROWS = 4;  // forward

// Tokens per wavefront (or workgroup, above WIDE features) and splits of a
// group's tokens in the backward pass.  A workgroup per CU and 2 rows per
// wavefront at least: more workgroups leave more partial sums (8192 tokens x
// 1152, bf16: 256 workgroups of eight wavefronts 19.0 us, 512 of eight 23.0, 512
// of four 19.2, 768 of four 20.0).  Two per CU for many rows of up to 256
// features, which are so short that latency counts (30798 x 191: 1 per CU 22, 2
// 18.0, 4 17.8 us; 20000 x 64 12.6, 11.3, 14.2; but 16000 x 512 17.7, 21 with 2,
// 9000 x 256 12.2, 12.6, and 5214 x 161 8.5, 10.1).
struct Split {
    int rows, splits;
};
Split grad_split(int B, int L, int C, int groups) {
    const long long group_rows = (long long)B * L / groups;
    const int block = C <= WIDE ? GRAD_ROWS : 1;
    const int slots = C <= 256 && (long long)B * L >= 16384 ? 512 : 256;
    long long splits = (slots + groups - 1) / groups;
    long long rows = (group_rows + splits * block - 1) / (splits * block);
    if (rows < 2) rows = 2;
    splits = (group_rows + rows * block - 1) / (rows * block);
    return Split{(int)rows, (int)splits};
}

template <bool F32, class S>
hipError_t run_norm(NormParams& p, hipStream_t stream) {
    // 16 wavefronts per CU (32768 tokens x 1152, fp32: 2048 in all 49.7 us, 4096 49.2, 16384 51.2)
    const long long units = 256 * 16 / S::WAVES;
    p.rows = (int)((p.M + units - 1) / units);
    const long long per_block = (long long)p.rows * S::ROWS;
    hipLaunchKernelGGL((norm_kernel<F32, S>), dim3((unsigned)((p.M + per_block - 1) / per_block)), dim3(S::NT), 0, stream, p);
    return hipGetLastError();
}

template <bool F32, class S>
hipError_t run_grad(NormParams& p, int groups, hipStream_t stream) {
    hipLaunchKernelGGL((norm_grad_kernel<F32, S>), dim3((unsigned)(groups * p.splits)), dim3(S::NT), 0, stream, p);
    return hipGetLastError();
}

// The narrowest shape that holds C features: vectors of 16 bytes of the wider
// of the two tensors, single elements below one vector.
template <int ROWS, bool EXACT, class F>
hipError_t by_width(int C, F&& run) {
    if (C <= 256) return run(Shape<4, 1, 1, ROWS, EXACT>{});
    if (C <= 512) return run(Shape<4, 2, 1, ROWS, EXACT>{});
    if (C <= WIDE) return run(Shape<4, 5, 1, ROWS, EXACT>{});
    if (C <= 2048) return run(Shape<4, 2, 4, ROWS, EXACT>{});
    if (C <= 4096) return run(Shape<4, 4, 4, ROWS, EXACT>{});
    if (C <= 8192) return run(Shape<4, 2, 16, ROWS, EXACT>{});
    return run(Shape<4, 4, 16, ROWS, EXACT>{});
}
template <int ROWS, class F>
hipError_t by_shape(int C, F&& run) {
    if (C < 4) return run(Shape<1, 1, 1, ROWS, true>{});
    return C % 4 ? by_width<ROWS, false>(C, run) : by_width<ROWS, true>(C, run);
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
    return by_shape<FORWARD_ROWS>(a.C, [&](auto s) {
        return a.x_f32 ? run_norm<true, decltype(s)>(p, stream) : run_norm<false, decltype(s)>(p, stream);
    });
}

hipError_t launch_layer_norm_backward(const NormGradLaunch& a, hipStream_t stream) {
    const Split split = grad_split(a.B, a.L, a.C, a.groups);
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
    const bool two = (a.dweight || a.dbias) && split.splits > 1;
    if (two) {
        p.partial = a.partial;
    } else {
        p.dweight = a.dweight;
        p.dbias = a.dbias;
    }
    const hipError_t e = by_shape<GRAD_ROWS>(a.C, [&](auto s) {
        return a.x_f32 ? run_grad<true, decltype(s)>(p, a.groups, stream) : run_grad<false, decltype(s)>(p, a.groups, stream);
    });
    if (e != hipSuccess || !two) return e;
    // 256 splits: 16 in flight take 0.6 to 1.1 us less than 4; 32 splits: 1.5 us more
    const auto sum = split.splits <= 64 ? norm_sum_kernel<4> : norm_sum_kernel<16>;
    hipLaunchKernelGGL(sum, dim3((2 * a.C + 63) / 64, a.groups), dim3(1024), 0, stream, a.partial, a.dweight, a.dbias, a.C,
                       split.splits);
    return hipGetLastError();
}

}  // namespace dfa
