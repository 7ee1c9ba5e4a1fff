// The linear layer for gfx950 (CDNA4): Y = residual + gate * act(X W^T + bias),
// fp32 from the accumulators to the one rounding of Y.
//
// The main loops are those of dfa_tiles.h; here are their output, the
// kernels for other cases, and the rule between them.
#include "dfa_epilogue.h"
#include "dfa_tiles.h"

namespace dfa {
namespace {

struct LinearParams : Operands {
    Rows gate;
    const void* residual;
    void* Y;
    int act_code;
};

// Output of one wavefront: block by block of 32 x 32 through its scratch (4 KB,
// chunk c of four features of token t at c ^ (t & 7)), so that a lane holds 16
// bytes of a row of Y and rows leave in order; stored straight from the
// accumulators, 4 bytes a lane, the same rows took 15% of the whole product
// longer.  The residual of DEPTH blocks is in flight ahead of the one that is
// formed, the first of them under the tile's last MFMAs.
template <bool F32, class T>
struct LinearOut {
    using Params = LinearParams;
    static constexpr int SCRATCH = 2 * 32 * 32;
    static constexpr bool FROM_BIAS = false;
    static constexpr int E = F32 ? 4 : 8, SZ = F32 ? 4 : 2;        // features of a lane, bytes of an element
    static constexpr int RPI = 2 * E, REPS = 32 / RPI;             // tokens per instruction, instructions per block
    static constexpr int BLOCKS = T::MB * T::NB, DEPTH = BLOCKS < 5 ? BLOCKS : 3;
    static_assert(T::STORES <= BLOCKS * REPS, "stores of a wavefront's output");
    u32x4 r[DEPTH][REPS];

    // residual of a block of a whole tile
    __device__ __forceinline__ void fetch(const LinearParams& p, int blk, int nw0, int tw0, int lane) {
        const int mb = blk / T::NB, nb = blk % T::NB, lt = lane / (32 / E), lf = lane % (32 / E) * E;
        const char* from = (const char*)p.residual + ((size_t)(tw0 + lt) * p.N + nw0 + lf) * SZ;
#pragma unroll
        for (int q = 0; q < REPS; ++q)
            __builtin_memcpy(&r[blk % DEPTH][q], from + (uint32_t)(32 * nb + RPI * q) * (uint32_t)p.N * SZ + 32 * mb * SZ, 16);
    }
    __device__ __forceinline__ void ahead(const LinearParams& p, int nw0, int tw0, int lane, bool whole) {
        if (!p.residual || !whole) return;
#pragma unroll
        for (int b = 0; b < DEPTH; ++b) fetch(p, b, nw0, tw0, lane);
    }
    template <bool WHOLE>
    __device__ __forceinline__ void store(const LinearParams& p, f32x16 (&acc)[T::MB][T::NB], uint16_t* scratch16, int nw0, int tw0,
                                          int lane) {
        // opaque: nothing of the addressing is to be kept in registers through the next tile's k loop
        asm volatile("" : "+v"(lane));
        float* scratch = (float*)scratch16;
        const int r32 = lane & 31, h = lane >> 5;
        const int lt = lane / (32 / E), lf = lane % (32 / E) * E;   // the lane's token and features
        const uint32_t rowb = (uint32_t)p.N * SZ;
        const size_t base = ((size_t)(tw0 + lt) * p.N + nw0 + lf) * SZ;
        char* out = (char*)p.Y + base;
        const char* res = (const char*)p.residual + base;
#pragma unroll
        for (int mb = 0; mb < T::MB; ++mb) {
            const int f = nw0 + 32 * mb + lf;
            float bias[E], g[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                bias[e] = p.bias && (WHOLE || f + e < p.N) ? p.bias[f + e] : 0.f;
                g[e] = p.gate.p && !p.gate.stride && (WHOLE || f + e < p.N) ? p.gate.p[f + e] : 1.f;
            }
            int entry = -1;
#pragma unroll
            for (int nb = 0; nb < T::NB; ++nb) {
                const int blk = mb * T::NB + nb;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *(f32x4*)(scratch + r32 * 32 + (((2 * i + h) ^ (r32 & 7)) << 2)) =
                        f32x4{acc[mb][nb][4 * i], acc[mb][nb][4 * i + 1], acc[mb][nb][4 * i + 2], acc[mb][nb][4 * i + 3]};
                __builtin_amdgcn_wave_barrier();   // the wavefront's LDS accesses complete in order
#pragma unroll
                for (int q = 0; q < REPS; ++q) {
                    const int tr = lt + RPI * q, t = tw0 + 32 * nb + tr;
                    const uint32_t at = (uint32_t)(32 * nb + RPI * q) * rowb + 32 * mb * SZ;
                    float z[E], x[E];
#pragma unroll
                    for (int c = 0; c < E / 4; ++c) {
                        const f32x4 v = *(const f32x4*)(scratch + tr * 32 + (((lf / 4 + c) ^ (tr & 7)) << 2));
#pragma unroll
                        for (int e = 0; e < 4; ++e) z[4 * c + e] = v[e] + bias[4 * c + e];
                    }
                    if (!WHOLE && (t >= p.M || f >= p.N)) continue;
                    const bool full = WHOLE || f + E <= p.N;
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = 0.f;
                    if (p.residual) {
                        if constexpr (WHOLE) {
                            const u32x4 v = r[blk % DEPTH][q];
#pragma unroll
                            for (int e = 0; e < E; ++e)
                                x[e] = __builtin_bit_cast(float, F32 ? v[e] : e & 1 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16);
                        } else if (full) {
                            read_row<F32, E>(x, res + at);
                        } else {
#pragma unroll
                            for (int e = 0; e < E; ++e) {
                                float one[1] = {0.f};
                                if (f + e < p.N) read_row<F32, 1>(one, res + at + e * SZ);
                                x[e] = one[0];
                            }
                        }
                    }
                    activate<E>(z, p.act_code);
                    if (p.gate.p && p.gate.stride) {
                        const int en = fast_div(t, p.lmul, p.lshift);
                        if (en != entry) {
                            entry = en;
                            const float* gp = p.gate.p + (size_t)en * p.gate.stride + f;
#pragma unroll
                            for (int e = 0; e < E; ++e)
                                if (WHOLE || f + e < p.N) g[e] = gp[e];
                        }
                    }
#pragma unroll
                    for (int e = 0; e < E; ++e) z[e] = fmaf(z[e], g[e], x[e]);
                    if (full) {
                        write_row<F32, E>(z, out + at);
                    } else {
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            float one[1] = {z[e]};
                            if (f + e < p.N) write_row<F32, 1>(one, out + at + e * SZ);
                        }
                    }
                }
                __builtin_amdgcn_wave_barrier();
                if (WHOLE && p.residual && blk + DEPTH < BLOCKS) fetch(p, blk + DEPTH, nw0, tw0, lane);
            }
        }
    }
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
    const uint16_t* xr = p.act;
    const int b = t / p.L;
    if (p.H == 1) xr += (size_t)t * p.K;
    else xr += ((size_t)b * p.H * p.L + (t - b * p.L)) * p.d;
    const uint16_t* wr = p.W + (size_t)min(n0 + row, p.N - 1) * p.K;
    const int wt = wave & 1, wf = wave >> 1;
    const int f = n0 + 32 * wf + r32;
    const float bias = p.bias ? p.bias[min(f, p.N - 1)] : 0.f;
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
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
        float z[1] = {acc[i] + bias}, r[1] = {0.f};
        const size_t o = ((size_t)tt * p.N + f) * (YF32 ? 4 : 2);
        if (p.residual) read_row<YF32, 1>(r, (const char*)p.residual + o);
        activate<1>(z, p.act_code);
        z[0] = fmaf(z[0], p.gate.p ? p.gate.p[(size_t)(tt / p.L) * p.gate.stride + f] : 1.f, r[0]);
        write_row<YF32, 1>(z, (char*)p.Y + o);
    }
}

// Tile shapes, features x tokens, as the projections take them (dfa_gemm.hip),
// with the same rule between them: 64 x 64 and 128 x 128 rings while one tile
// per CU covers the output, else 128 x 128 or 192 x 256 by the rounds they need.
// Block order: the 32 or 64 workgroups that an XCD has resident share the lines
// of their tiles in its L2; the fewest lines are in flight where they cover
// about as many tokens as features.  Groups of 3 token tiles of 256 (measured
// 1, 2, 3, 4, 8: 4096 x 1152 -> 4608 127, 126, 122, 130, 128 us; 32768 x 4608
// -> 1152 365, 366, 372, 369, 378; 32768 x 1152 -> 4608 381, 378, 367, 379,
// 388) and of 4 of 128 (1, 4, 8: 8192 x 1152 -> 4608 139, 136, 146).
using Tile64 = Tile<1, 1, 2, 2, 2, 4>;
using Tile128Ring = Tile<2, 1, 2, 4, 1, 4>;
using Tile128 = Tile<2, 2, 2, 2, 2>;
using Tile192 = Tile<3, 2, 2, 4, 1>;

template <int ACT, bool F32>
hipError_t launch_tiles(LinearParams& p, hipStream_t stream) {
    p.group = 4;
    if (tiles<Tile64>(p) <= 256) return launch_shape<ACT, LinearOut<F32, Tile64>, Tile64>(p, stream);
    const long long n128 = tiles<Tile128>(p), n192 = tiles<Tile192>(p);
    if (n128 <= 256) return launch_shape<ACT, LinearOut<F32, Tile128Ring>, Tile128Ring>(p, stream);
    const long long last = n128 % 512;
    const long long rounds128 = 100 * (n128 / 512) + (last == 0 ? 0 : (last <= 256 ? 65 : 100));
    const long long rounds192 = 125 * ((n192 + 255) / 256);
    if (rounds192 >= rounds128) return launch_shape<ACT, LinearOut<F32, Tile128>, Tile128>(p, stream);
    p.group = 3;
    return launch_shape<ACT, LinearOut<F32, Tile192>, Tile192>(p, stream);
}

template <bool F32>
hipError_t launch(LinearParams& p, hipStream_t stream) {
    if (p.H > 1 && p.K % (2 * GK) == 0) return launch_tiles<ACT_HEADS, F32>(p, stream);
    if (p.H == 1 && p.K % (2 * GK) == 0) return launch_tiles<ACT_ROWS, F32>(p, stream);
    if (p.H == 1 && p.K % 8 == 0) return launch_tiles<ACT_ROWS_TAIL, F32>(p, stream);
    p.nft = (p.N + 63) / 64;
    p.ntt = (p.M + 63) / 64;
    const long long blocks = (long long)p.nft * p.ntt;
    if (blocks > (1LL << 23)) return hipErrorInvalidValue;
    hipLaunchKernelGGL(linear_general_kernel<F32>, dim3((unsigned)blocks), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear(const LinearLaunch& a, hipStream_t stream) {
    LinearParams p{};
    p.W = (const uint16_t*)a.W;
    p.act = (const uint16_t*)a.X;
    p.bias = a.bias;
    p.L = a.L;
    p.H = a.H;
    p.d = a.K / a.H;
    p.M = a.B * a.L;
    p.K = a.K;
    p.N = a.N;
    p.gate = a.gate;
    p.residual = a.residual;
    p.Y = a.Y;
    p.act_code = a.act;
    return a.y_f32 ? launch<true>(p, stream) : launch<false>(p, stream);
}

}  // namespace dfa
