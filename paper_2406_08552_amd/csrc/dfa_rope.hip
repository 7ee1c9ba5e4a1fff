// Rotary positions over several axes for gfx950 (CDNA4): pair (x, y) of a head
// turns by theta = pos[token][axis] base^(-2 i / n), to
// (x cos - y sin, x sin + y cos); the inverse turns by -theta.
//
// An HBM stream of Q and K.  A lane owns some dims of one token (so that an
// output may replace its input) and walks the heads with them: their angles
// are formed once for all heads of Q and K that the lane visits.  The angle is
// reduced in fp64, in revolutions, because a position of thousands times a
// frequency near 1 leaves fp32 few bits of the fraction; sine and cosine of
// the fraction are v_sin_f32 and v_cos_f32, off by at most 1.25e-7 over 2^22
// fractions of -1/2 to 1/2.
//
// 16 heads of d = 72 at 2 x 16384 tokens, halves, take 59 us for Q and K, 302 MB
// at 5.1 TB/s, the rate of a large copy; at 2 x 6480 tokens, pairs, 25 us (4.8 TB/s).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "dfa_internal.h"

namespace dfa {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256, WAVES = THREADS / 64;
// heads whose loads a lane has in flight (2, 4, 8, d = 72, 16 heads of Q and of K: 2048
// tokens 8.8, 8.3, 9.4 us; 32768 60, 60, 66)
constexpr int BATCH = 4;
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
    int sections[ROPE_AXES_MAX];   // 0 behind the last
    double log2_base;
    bool interleaved, inverse;
};

__device__ __forceinline__ float bf16_at(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// What a head's dims turn by, formed by the workgroup (a lane per dim: a table
// among the kernel's arguments, read by every wavefront, took longer): a dim
// becomes x cos(phi) + partner sin(phi) with phi = pos[axis] * 2 pi turn, where
// turn is -base^(-2 i / n) / (2 pi) for the first of a pair, + for the second.
struct Dims {
    double turn[ROPE_D_MAX];
    uint8_t axis[ROPE_D_MAX], partner[ROPE_D_MAX];
    uint8_t lo[ROPE_D_MAX / 2];    // halves: the first of the pairs, in order
    __device__ __forceinline__ void form(const RopeParams& p) {
        static_assert(THREADS >= ROPE_D_MAX, "a lane per dim");
        const int x = threadIdx.x;
        if (x < p.d) {
            // the section of x; the dims behind the last are one that does not turn
            int o = 0, n = 0, s = KEEP, at = 0;
#pragma unroll
            for (int a = 0; a < ROPE_AXES_MAX; ++a) {
                if (x >= at && x < at + p.sections[a]) {
                    o = at;
                    n = p.sections[a];
                    s = a;
                }
                at += p.sections[a];
            }
            if (s == KEEP) {
                o = at;
                n = p.d - at;
            }
            const int i = x - o, half = n / 2;
            const bool first = p.interleaved ? i % 2 == 0 : i < half;
            const int pair = p.interleaved ? i / 2 : first ? i : i - half;
            // 1 / (2 pi) turns per radian
            const double t = s == KEEP ? 0.0 : 0.15915494309189533577 * exp2(-p.log2_base * (double)pair / (double)half);
            turn[x] = first != p.inverse ? -t : t;
            axis[x] = (uint8_t)s;
            partner[x] = (uint8_t)(p.interleaved ? x ^ 1 : first ? x + half : x - half);
            if (first) lo[o / 2 + pair] = (uint8_t)x;
        }
        // LDS alone: __syncthreads() would also wait for the loads in flight
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    }
};

// Positions of token l, and cosine and sine of one dim's angle.
struct Angles {
    float pos[ROPE_AXES_MAX];
    __device__ __forceinline__ Angles(const RopeParams& p, int b, long long l) {
        const float* at = p.pos + (size_t)b * p.pos_stride + (size_t)l * p.naxes;
#pragma unroll
        for (int a = 0; a < ROPE_AXES_MAX; ++a) pos[a] = a < p.naxes ? at[a] : 0.f;
    }
    __device__ __forceinline__ float along(int axis) const {
        return axis == 0 ? pos[0] : axis == 1 ? pos[1] : axis == 2 ? pos[2] : pos[3];
    }
    __device__ __forceinline__ void of(double turn, float x, float& c, float& s) const {
        const double rev = (double)x * turn;
        const float f = (float)(rev - rint(rev));
        s = __builtin_amdgcn_sinf(f);
        c = __builtin_amdgcn_cosf(f);
    }
};

// Offset, in elements, of the row of head h (Q's heads, then K's) of token l.
__device__ __forceinline__ size_t row_of(const RopeParams& p, int b, int h, long long l, int& which) {
    which = h >= p.heads[0];
    return (((size_t)b * p.heads[which] + (which ? h - p.heads[0] : h)) * p.L + l) * p.d;
}

enum { PAIRS, HALVES_EVEN, HALVES };   // partners: beside each other; pairs of dims in the other half; any dim

// d % 8 = 0: a lane owns eight neighbouring dims, 16 bytes.  Halves: their
// partners come from other lanes of the wavefront through LDS, by fours or (odd
// halves) by twos of bytes; loads of a unit's own two parts, 4 bytes each at
// d = 72 in sections of 36, took 76 us where this takes 59 (302 MB moved).
template <int EX>
__global__ void __launch_bounds__(THREADS) rope_rows_kernel(RopeParams p) {
    __shared__ u32x4 xch[EX == PAIRS ? 1 : WAVES][EX == PAIRS ? 1 : BATCH][64];
    __shared__ Dims dims;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per_wave = p.tokens / WAVES;
    const int lt = lane / p.units, d0 = 8 * (lane - lt * p.units);
    const bool mine = lt < per_wave;
    const int nh = p.heads[0] + p.heads[1];
    const int h0 = blockIdx.y * p.per_block, h1 = min(nh, h0 + p.per_block);
    bool formed = false;
    double turn[8];
    int from[8];   // byte offset of the partner in the wavefront's rows
    // Where the sections end: a dim's axis by comparison, not by another LDS
    // read of the turns (2048 tokens x 32 heads: 8.4 and 7.6 us).
    int end[ROPE_AXES_MAX];
#pragma unroll
    for (int a = 0; a < ROPE_AXES_MAX; ++a) end[a] = (a ? end[a - 1] : 0) + p.sections[a];
    const int turning = end[ROPE_AXES_MAX - 1] - d0;   // of the lane's dims, those that turn
    for (int b = blockIdx.z; b < p.B; b += gridDim.z)
        // every wavefront of the workgroup makes the same number of rounds
        for (long long t0 = (long long)blockIdx.x * p.tokens; t0 < p.L; t0 += (long long)gridDim.x * p.tokens) {
            const long long l = t0 + wave * per_wave + lt;
            const bool in = mine && l < p.L;
            u32x4 next[BATCH];
            auto load = [&](int h) {
#pragma unroll
                for (int j = 0; j < BATCH; ++j)
                    if (in && h + j < h1) {
                        int which;
                        const size_t row = row_of(p, b, h + j, l, which);
                        next[j] = *(const u32x4*)(p.in[which] + 2 * (row + d0));
                    }
            };
            // in flight while the turns are formed: the positions, and the first heads
            const Angles ang(p, b, in ? l : t0);
            load(h0);
            if (!formed) {
                formed = true;
                dims.form(p);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    turn[i] = dims.turn[d0 + i];
                    from[i] = 2 * (lt * p.d + (i < turning ? dims.partner[d0 + i] : d0 + i));
                }
            }
            float cs[8], sn[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (EX == PAIRS && i % 2) {   // the second of a pair turns by the same angle
                    cs[i] = cs[i - 1];
                    sn[i] = -sn[i - 1];
                } else {
                    const int x = d0 + i;
                    ang.of(turn[i], ang.along(x < end[0] ? 0 : x < end[1] ? 1 : x < end[2] ? 2 : 3), cs[i], sn[i]);
                }
            }
            for (int h = h0; h < h1; h += BATCH) {
                u32x4 x[BATCH];
#pragma unroll
                for (int j = 0; j < BATCH; ++j) x[j] = next[j];
                if (h + BATCH < h1) load(h + BATCH);
                if constexpr (EX != PAIRS) {
#pragma unroll
                    for (int j = 0; j < BATCH; ++j) xch[wave][j][lane] = x[j];
                    __builtin_amdgcn_wave_barrier();   // the wavefront's LDS accesses complete in order
                }
#pragma unroll
                for (int j = 0; j < BATCH; ++j) {
                    if (!in || h + j >= h1) continue;
                    const char* rows = (const char*)xch[EX == PAIRS ? 0 : wave][EX == PAIRS ? 0 : j];
                    u32x4 y;
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const uint32_t u = x[j][i / 2];
                        uint32_t q;
                        if constexpr (EX == PAIRS) q = u << 16 | u >> 16;
                        else if constexpr (EX == HALVES_EVEN) q = *(const uint32_t*)(rows + from[i]);
                        else q = *(const uint16_t*)(rows + from[i]) | (uint32_t) * (const uint16_t*)(rows + from[i + 1]) << 16;
                        const float a = fmaf(bf16_at((uint16_t)u), cs[i], bf16_at((uint16_t)q) * sn[i]);
                        const float c = fmaf(bf16_at(u >> 16), cs[i + 1], bf16_at(q >> 16) * sn[i + 1]);
                        const uint32_t r = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)c});
                        y[i / 2] = i < turning ? r : u;   // sections are even
                    }
                    int which;
                    const size_t row = row_of(p, b, h + j, l, which);
                    *(u32x4*)(p.out[which] + 2 * (row + d0)) = y;
                }
                if constexpr (EX != PAIRS) __builtin_amdgcn_wave_barrier();
            }
        }
}

// Other head dims: U pairs per lane.  INTER: 2 U consecutive elements; else U at lo and U at their partners.
template <bool INTER, int U>
__global__ void __launch_bounds__(THREADS) rope_units_kernel(RopeParams p) {
    __shared__ Dims dims;
    dims.form(p);
    const int lt = threadIdx.x / p.units, u = threadIdx.x - lt * p.units;
    if (lt >= p.tokens) return;
    const int lo = INTER ? 2 * U * u : dims.lo[U * u], hi = INTER ? lo + U : dims.partner[lo];
    const int nh = p.heads[0] + p.heads[1];
    const int h0 = blockIdx.y * p.per_block, h1 = min(nh, h0 + p.per_block);
    for (int b = blockIdx.z; b < p.B; b += gridDim.z)
        for (long long l = (long long)blockIdx.x * p.tokens + lt; l < p.L; l += (long long)gridDim.x * p.tokens) {
            float cs[U], sn[U];
            bool keep[U];
            const Angles ang(p, b, l);
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int first = lo + (INTER ? 2 * i : i);
                keep[i] = dims.axis[first] == KEEP;
                ang.of(dims.turn[first], ang.along(dims.axis[first]), cs[i], sn[i]);
            }
            for (int h = h0; h < h1; h += BATCH) {
                uint16_t x[BATCH][2 * U];
#pragma unroll
                for (int j = 0; j < BATCH; ++j)
                    if (h + j < h1) {
                        int which;
                        const size_t row = row_of(p, b, h + j, l, which);
                        __builtin_memcpy(x[j], p.in[which] + 2 * (row + lo), 2 * U);
                        __builtin_memcpy(x[j] + U, p.in[which] + 2 * (row + hi), 2 * U);
                    }
#pragma unroll
                for (int j = 0; j < BATCH; ++j) {
                    if (h + j >= h1) break;
#pragma unroll
                    for (int i = 0; i < U; ++i) {
                        uint16_t &s = x[j][INTER ? 2 * i : i], &t = x[j][INTER ? 2 * i + 1 : U + i];
                        const float xs = bf16_at(s), xt = bf16_at(t);
                        const uint16_t ys = to_bf16(fmaf(xs, cs[i], xt * sn[i])), yt = to_bf16(fmaf(xt, cs[i], -(xs * sn[i])));
                        s = keep[i] ? s : ys;
                        t = keep[i] ? t : yt;
                    }
                    int which;
                    const size_t row = row_of(p, b, h + j, l, which);
                    __builtin_memcpy(p.out[which] + 2 * (row + lo), x[j], 2 * U);
                    __builtin_memcpy(p.out[which] + 2 * (row + hi), x[j] + U, 2 * U);
                }
            }
        }
}

// Grid of a kernel whose workgroups take p.tokens tokens.
dim3 grid_of(RopeParams& p) {
    const int nh = p.heads[0] + p.heads[1];
    const long long tiles = ((long long)p.L + p.tokens - 1) / p.tokens;
    // 2048 workgroups at least: fewer heads each, down to one batch of loads (1024, 2048, 4096, 16 heads of Q and of K:
    // 12960 tokens 27.9, 25.9, 28.1 us; 32768 65, 61, 60)
    long long parts = (2047 + tiles * p.B) / (tiles * p.B);
    if (parts > (nh + BATCH - 1) / BATCH) parts = (nh + BATCH - 1) / BATCH;
    if (parts > 65535) parts = 65535;
    p.per_block = (int)((nh + parts - 1) / parts);
    p.per_block = (p.per_block + BATCH - 1) / BATCH * BATCH;
    parts = (nh + p.per_block - 1) / p.per_block;
    return dim3((unsigned)(tiles < (1 << 22) ? tiles : (1 << 22)), (unsigned)parts, p.B < 65535 ? p.B : 65535);
}

template <int EX>
hipError_t run_rows(RopeParams& p, hipStream_t stream) {
    p.units = p.d / 8;
    p.tokens = WAVES * (64 / p.units);
    const dim3 grid = grid_of(p);
    hipLaunchKernelGGL((rope_rows_kernel<EX>), grid, dim3(THREADS), 0, stream, p);
    return hipGetLastError();
}

template <bool INTER, int U>
hipError_t run_units(RopeParams& p, hipStream_t stream) {
    p.units = p.d / (2 * U);
    p.tokens = THREADS / p.units;
    const dim3 grid = grid_of(p);
    hipLaunchKernelGGL((rope_units_kernel<INTER, U>), grid, dim3(THREADS), 0, stream, p);
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
    p.log2_base = log2(a.base);
    p.interleaved = a.interleaved;
    p.inverse = a.inverse;
    bool even = true;   // every half a whole number of two dims
    int rest = a.d;
    for (int i = 0; i < a.naxes; ++i) {
        p.sections[i] = a.sections[i];
        even = even && a.sections[i] % 4 == 0;
        rest -= a.sections[i];
    }
    if (a.d % 8 == 0) {
        if (a.interleaved) return run_rows<PAIRS>(p, stream);
        return even ? run_rows<HALVES_EVEN>(p, stream) : run_rows<HALVES>(p, stream);
    }
    // two pairs to a lane where that divides the head's pairs (halves: every section's, and the rest's)
    const int U = a.d % 4 == 0 && (a.interleaved || (even && rest % 4 == 0)) ? 2 : 1;
    if (a.interleaved) return U == 2 ? run_units<true, 2>(p, stream) : run_units<true, 1>(p, stream);
    return U == 2 ? run_units<false, 2>(p, stream) : run_units<false, 1>(p, stream);
}

}  // namespace dfa
