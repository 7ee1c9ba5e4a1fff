// Rotary positions over several axes for gfx950 (CDNA4): pair (x, y) of a head
// turns by theta = pos[token][axis] base^(-2 i / n), to
// (x cos - y sin, x sin + y cos); the inverse turns by -theta.
//
// An HBM stream of Q and K.  A lane owns some pairs of one token (so that an
// output may replace its input) and walks the heads with them: their angles
// are formed once for all heads of Q and K that the lane visits.  The angle is
// reduced in fp64, in revolutions, because a position of thousands times a
// frequency near 1 leaves fp32 few bits of the fraction.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "dfa_internal.h"

namespace dfa {
namespace {

constexpr int THREADS = 256;
constexpr int BATCH = 4;        // heads whose loads a lane has in flight
constexpr uint8_t KEEP = 255;   // "axis" of the dims behind the last section

struct RopeParams {
    const char* in[2];       // Q, K
    char* out[2];
    int heads[2];
    const float* pos;
    long long pos_stride;
    int naxes;
    int B, L, d;
    int units;               // lanes per token
    int tokens;              // per workgroup
    int per_block;           // heads that one workgroup visits
    float sign;
    double freq[ROPE_D_MAX / 2];    // per pair: base^(-2 i / n) / (2 pi)
    uint8_t axis[ROPE_D_MAX / 2];   // and its axis, or KEEP
    uint8_t lo[ROPE_D_MAX / 2];     // per unit of halves: first dim of its first elements,
    uint8_t hi[ROPE_D_MAX / 2];     // and of their partners
};

__device__ __forceinline__ float bf16_at(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// U pairs per lane: INTER, 2 U consecutive elements; else U at lo and U at hi.
template <bool INTER, int U>
__global__ void __launch_bounds__(THREADS) rope_kernel(RopeParams p) {
    const int lt = threadIdx.x / p.units, u = threadIdx.x - lt * p.units;
    if (lt >= p.tokens) return;
    const int lo = INTER ? 2 * U * u : p.lo[u], hi = INTER ? lo + U : p.hi[u];
    const int nh = p.heads[0] + p.heads[1];
    const int h0 = blockIdx.y * p.per_block, h1 = min(nh, h0 + p.per_block);
    for (int b = blockIdx.z; b < p.B; b += gridDim.z)
        for (long long l = (long long)blockIdx.x * p.tokens + lt; l < p.L; l += (long long)gridDim.x * p.tokens) {
            float cs[U], sn[U];
            bool keep[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int a = p.axis[u * U + i];
                keep[i] = a == KEEP;
                const float pos = keep[i] ? 0.f : p.pos[(size_t)b * p.pos_stride + (size_t)l * p.naxes + a];
                const double rev = (double)pos * p.freq[u * U + i];
                sincospif(2.f * (float)(rev - rint(rev)), &sn[i], &cs[i]);
                sn[i] *= p.sign;
            }
            for (int h = h0; h < h1; h += BATCH) {
                uint16_t x[BATCH][2 * U];
                size_t at[BATCH];
#pragma unroll
                for (int j = 0; j < BATCH; ++j) {
                    const int which = h + j >= p.heads[0], hw = which ? h + j - p.heads[0] : h + j;
                    at[j] = (((size_t)b * p.heads[which] + hw) * p.L + l) * p.d * 2;
                    if (h + j < h1) {
                        __builtin_memcpy(x[j], p.in[which] + at[j] + 2 * lo, 2 * U);
                        __builtin_memcpy(x[j] + U, p.in[which] + at[j] + 2 * hi, 2 * U);
                    }
                }
#pragma unroll
                for (int j = 0; j < BATCH; ++j) {
                    if (h + j >= h1) break;
#pragma unroll
                    for (int i = 0; i < U; ++i) {
                        uint16_t &s = x[j][INTER ? 2 * i : i], &t = x[j][INTER ? 2 * i + 1 : U + i];
                        const float xs = bf16_at(s), xt = bf16_at(t);
                        const uint16_t ys = to_bf16(xs * cs[i] - xt * sn[i]), yt = to_bf16(xs * sn[i] + xt * cs[i]);
                        s = keep[i] ? s : ys;
                        t = keep[i] ? t : yt;
                    }
                    char* out = p.out[h + j >= p.heads[0]] + at[j];
                    __builtin_memcpy(out + 2 * lo, x[j], 2 * U);
                    __builtin_memcpy(out + 2 * hi, x[j] + U, 2 * U);
                }
            }
        }
}

template <bool INTER, int U>
hipError_t run(RopeParams& p, hipStream_t stream) {
    p.units = p.d / (2 * U);
    p.tokens = THREADS / p.units;
    const int nh = p.heads[0] + p.heads[1];
    const long long tiles = ((long long)p.L + p.tokens - 1) / p.tokens;
    // few workgroups: fewer heads each, down to one batch of loads
    long long parts = (2048 + tiles * p.B - 1) / (tiles * p.B);
    if (parts > (nh + BATCH - 1) / BATCH) parts = (nh + BATCH - 1) / BATCH;
    if (parts > 65535) parts = 65535;
    p.per_block = (int)((nh + parts - 1) / parts);
    parts = (nh + p.per_block - 1) / p.per_block;
    const unsigned gx = (unsigned)(tiles < (1 << 22) ? tiles : (1 << 22)), gz = p.B < 65535 ? p.B : 65535;
    hipLaunchKernelGGL((rope_kernel<INTER, U>), dim3(gx, (unsigned)parts, gz), dim3(THREADS), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeLaunch& a, hipStream_t stream) {
    RopeParams p{};
    p.in[0] = (const char*)a.Q;
    p.in[1] = (const char*)a.K;
    p.out[0] = (char*)a.Qout;
    p.out[1] = (char*)a.Kout;
    p.heads[0] = a.Hq;
    p.heads[1] = a.Hk;
    p.pos = a.pos;
    p.pos_stride = a.pos_stride;
    p.naxes = a.naxes;
    p.B = a.B;
    p.L = a.L;
    p.d = a.d;
    p.sign = a.inverse ? -1.f : 1.f;
    // The pairs of every section in turn, then those of the dims that stay; one
    // power per axis, the frequencies by multiplication.  U pairs go to a lane:
    // as many (a 16-byte access at most) as divide every section's halves, or
    // the head's pairs where they lie side by side.
    int U = a.interleaved ? 4 : 8, n = 0, o = 0;
    uint8_t first[ROPE_D_MAX / 2], partner[ROPE_D_MAX / 2];
    for (int s = 0; s <= a.naxes; ++s) {
        const int half = (s < a.naxes ? a.sections[s] : a.d - o) / 2;
        const double ratio = s < a.naxes ? pow(a.base, -1.0 / half) : 0.0;
        double f = s < a.naxes ? 0.15915494309189533577 : 0.0;   // 1 / (2 pi)
        for (int i = 0; i < half; ++i, ++n) {
            p.freq[n] = f;
            p.axis[n] = s < a.naxes ? (uint8_t)s : KEEP;
            first[n] = (uint8_t)(o + i);
            partner[n] = (uint8_t)(o + half + i);
            f *= ratio;
        }
        o += 2 * half;
        while (!a.interleaved && half % U) U /= 2;
    }
    while (n % U) U /= 2;
    for (int u = 0; u * U < n; ++u) {
        p.lo[u] = first[u * U];
        p.hi[u] = partner[u * U];
    }
    if (a.interleaved) {
        if (U == 4) return run<true, 4>(p, stream);
        if (U == 2) return run<true, 2>(p, stream);
        return run<true, 1>(p, stream);
    }
    if (U == 8) return run<false, 8>(p, stream);
    if (U == 4) return run<false, 4>(p, stream);
    if (U == 2) return run<false, 2>(p, stream);
    return run<false, 1>(p, stream);
}

}  // namespace dfa
