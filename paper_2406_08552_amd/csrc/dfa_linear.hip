// The linear layer for gfx950 (CDNA4): Y = residual + gate * act(X W^T + bias),
// fp32 from the accumulators to the one rounding of Y.
//
// The main loops are those of dfa_tiles.h; here are their output, the
// kernels for other cases, and the rule between them.  Few tokens are a stream
// of the weights (2 x 1152 -> 6912 5.8 us, of which a launch takes 3.3).  Many
// are bound by the copies of the k-tiles into LDS and the clock that power
// leaves: 8192 x 1152 -> 4608 with GELU's tanh form 110 us (789 TFLOP/s), 32768 x
// 4608 -> 1152 with gate and fp32 residual 370 us (940 TFLOP/s), 302 MB of
// residual and output among it, which move beside the next tile's products.
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
    static constexpr int BLOCKS = T::MB * T::NB, DEPTH = BLOCKS < 5 ? BLOCKS : BLOCKS < 8 ? 3 : 2;
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
                    if (p.gate.p || p.residual) {
#pragma unroll
                        for (int e = 0; e < E; ++e) z[e] = fmaf(z[e], g[e], x[e]);
                    }
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

// Element k of token t of the activations, k a multiple of 8 (heads: a chunk of
// eight lies in one, since d % 8 = 0).
struct TokenRow {
    const uint16_t* p;
    long long head;   // elements from a head's dims on to the next head's, less d
    __device__ __forceinline__ TokenRow(const LinearParams& q, int t) {
        if (q.H == 1) {
            p = q.act + (size_t)t * q.K;
            head = 0;
        } else {
            const int b = fast_div(t, q.lmul, q.lshift);
            p = q.act + ((size_t)t + (size_t)b * (q.H - 1) * q.L) * q.d;
            head = (long long)(q.L - 1) * q.d;
        }
    }
    __device__ __forceinline__ const uint16_t* at(const LinearParams& q, int k) const {
        return head ? p + k + fast_div(k, q.dmul, q.dshift) * head : p + k;
    }
};

// Any K: rows that 16 bytes do not divide take no direct copies, so the k-tiles
// pass through registers, the next one in flight while this one is multiplied.
template <bool F32, class T>
__global__ void __launch_bounds__(T::NT) linear_any_kernel(LinearParams p) {
    constexpr int CH = (T::TF + T::TT) * 8 / T::NT;   // chunks of eight k per lane and k-tile
    using Out = LinearOut<F32, T>;
    __shared__ __attribute__((aligned(16))) uint16_t st[2][T::STAGE];
    __shared__ __attribute__((aligned(16))) uint16_t scratch[T::NW * Out::SCRATCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wf = wave % T::WF, wt = wave / T::WF, r32 = lane & 31, h = lane >> 5;
    const int row = tid >> 3, ch = tid & 7;           // and the rows NT / 8 apart
    const int ao = chunk_off(32 * T::MB * wf + r32, h), bo = chunk_off(T::TF + 32 * T::NB * wt + r32, h);
    const int nk = (p.K + GK - 1) / GK;
    // a contiguous range of tiles per XCD, as in gemm_stream_kernel
    const int x = blockIdx.x & 7, q = p.nblocks >> 3, rem = p.nblocks & 7;
    const int end = (x + 1) * q + min(x + 1, rem), stride = ((int)gridDim.x + 7 - x) >> 3;
    for (int blk = x * q + min(x, rem) + ((int)blockIdx.x >> 3); blk < end; blk += stride) {
        int n0, t0;
        tile_origin<T>(p, blk, n0, t0);
        u32x4 v[CH];
        auto load = [&](int k0) {
            const int k = k0 + 8 * ch;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int r = row + i * (T::NT / 8);
                v[i] = u32x4{0, 0, 0, 0};
                if (k < p.K) {
                    const uint16_t* from = r < T::TF ? p.W + (size_t)min(n0 + r, p.N - 1) * p.K
                                                     : p.act + (size_t)min(t0 + r - T::TF, p.M - 1) * p.K;
                    v[i] = load8(from + k, p.K - k);
                }
            }
        };
        f32x16 acc[T::MB][T::NB];
        zero_acc<T>(acc);
        load(0);
        for (int kt = 0; kt < nk; ++kt) {
            uint16_t* cur = st[kt & 1];
#pragma unroll
            for (int i = 0; i < CH; ++i) *(u32x4*)(cur + chunk_off(row + i * (T::NT / 8), ch)) = v[i];
            __syncthreads();   // behind it every wavefront has read the k-tile before this one
            if (kt + 1 < nk) load((kt + 1) * GK);
            Frag<T> f;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                f.read(cur, ks, ao, bo);
                mma<T, 0, T::MB * T::NB>(acc, f);
            }
        }
        const bool whole = n0 + T::TF <= p.N && t0 + T::TT <= p.M;
        const int nw0 = n0 + 32 * T::MB * wf, tw0 = t0 + 32 * T::NB * wt;
        Out out;
        out.ahead(p, nw0, tw0, lane, whole);
        if (whole) out.template store<true>(p, acc, scratch + wave * Out::SCRATCH, nw0, tw0, lane);
        else out.template store<false>(p, acc, scratch + wave * Out::SCRATCH, nw0, tw0, lane);
        __syncthreads();       // the last k-tile has been read, too
    }
}

// Few tokens: the weights' stream from HBM counts.  Few outputs: the length of K.
// A workgroup takes 16 features of 16 TB tokens; its wavefronts take the 64-element pieces of K in turn,
// straight into registers (16 features x 128 bytes, AHEAD pieces in flight),
// through v_mfma_f32_16x16x32_bf16 (A element e = A[l % 16][8 (l / 16) + e], B
// alike, output element i = D[4 (l / 16) + i][l % 16]), and add up in LDS.
template <bool F32, int TB>
__global__ void __launch_bounds__(512) linear_few_kernel(LinearParams p) {
    constexpr int NW = 8, AHEAD = TB > 1 ? 2 : 3;
    __shared__ float sums[NW][TB][16][17];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, kq = 8 * (lane >> 4), n0 = 16 * blockIdx.x, t0 = 16 * TB * blockIdx.y;
    const uint16_t* w = p.W + (size_t)min(n0 + r, p.N - 1) * p.K;
    f32x4 acc[TB];
#pragma unroll
    for (int tb = 0; tb < TB; ++tb) acc[tb] = f32x4{0.f, 0.f, 0.f, 0.f};
    u32x4 wv[AHEAD][2], xv[AHEAD][2][TB];
    auto load = [&](int slot, int k0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int k = k0 + 32 * i + kq;
            wv[slot][i] = u32x4{0, 0, 0, 0};
            if (k < p.K) wv[slot][i] = load8(w + k, p.K - k);
#pragma unroll
            for (int tb = 0; tb < TB; ++tb) {
                xv[slot][i][tb] = u32x4{0, 0, 0, 0};
                if (k < p.K) xv[slot][i][tb] = load8(TokenRow(p, min(t0 + 16 * tb + r, p.M - 1)).at(p, k), p.K - k);
            }
        }
    };
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) load(s, (wave + s * NW) * 64);
    for (int k0 = wave * 64; k0 < p.K; k0 += AHEAD * NW * 64) {
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {   // pieces behind the end are zeros
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int tb = 0; tb < TB; ++tb)
                    acc[tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, xv[s][i][tb]),
                                                                      __builtin_bit_cast(bf16x8, wv[s][i]), acc[tb], 0, 0, 0);
            load(s, k0 + (AHEAD + s) * NW * 64);
        }
    }
#pragma unroll
    for (int tb = 0; tb < TB; ++tb)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[wave][tb][4 * (lane >> 4) + i][r] = acc[tb][i];
    __syncthreads();
    for (int e = threadIdx.x; e < TB * 256; e += 512) {
        const int lt = e >> 4, t = t0 + lt, f = n0 + (e & 15);
        if (t >= p.M || f >= p.N) continue;
        float z[1] = {0.f}, x[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NW; ++i) z[0] += sums[i][lt >> 4][lt & 15][e & 15];
        if (p.bias) z[0] += p.bias[f];
        const size_t o = ((size_t)t * p.N + f) * (F32 ? 4 : 2);
        if (p.residual) read_row<F32, 1>(x, (const char*)p.residual + o);
        activate<1>(z, p.act_code);
        const float g = p.gate.p ? p.gate.p[(size_t)fast_div(t, p.lmul, p.lshift) * p.gate.stride + f] : 1.f;
        z[0] = fmaf(z[0], g, x[0]);
        write_row<F32, 1>(z, (char*)p.Y + o);
    }
}

// Tile shapes, features x tokens, and the rule between them:
//   64 x 64, ring      while two such tiles per CU cover the output, which a CU
//                      holds at once (us against the next: 602 x 1152 -> 1152 7.0
//                      and 12.4, 1790 x 1152 -> 1152 11.6 and 13.2, 1024 x 4608 ->
//                      1152 39 and 46; with more tiles 2000 x 1152 -> 1152 15.4, 13.3)
//   128 x 128, ring    while one per CU does (2000 x 1152 -> 1152 13.3, stream 16.7;
//                      3600 x 1152 -> 1152 25.1, stream 19.2); beyond, by the
//                      rounds that each needs:
//   128 x 128, stream  two workgroups per CU; a last round of one takes 0.65
//   192 x 256, stream  1.38 of its round for 1.5 of its output
//   256 x 256, stream  1.76 for 2, K a multiple of 128 (the others' registers
//                      spill); nothing runs beside a single round's output, which
//                      counts the more the fewer k-tiles there are (by 256 and 128, fp32
//                      residual: 12960 x 1152 -> 1152 70, 64 us, 6000 x 1152 -> 2304 66,
//                      66, 6000 x 2304 -> 2304 93, 98, 6000 x 4608 -> 2304 140, 151;
//                      bf16: 8000 x 1152 -> 1664 44, 48, 12000 x 1920 -> 1152 69, 78)
// us by 128, 192, 256: 32768 x 1152 -> 4608 396, 364, 342; 32768 x 4608 -> 1152
// 360, 330, 353; 8192 x 1152 -> 4608 105, 103, 109.
// Block order: the 32 or 64 workgroups that an XCD has resident share the lines
// of their tiles in its L2; the fewest lines are in flight where they cover
// about as many tokens as features.  Groups of 3 token tiles of 256 (measured
// 1, 2, 3, 4, 8: 8192 x 1152 -> 4608 127, 126, 122, 130, 128 us; 32768 x 4608
// -> 1152 365, 366, 372, 369, 378; 32768 x 1152 -> 4608 381, 378, 367, 379,
// 388) and of 4 of 128 (1, 4, 8: 8192 x 1152 -> 4608 139, 136, 146).
using Tile64 = Tile<1, 1, 2, 2, 2, 4>;
using Tile128Ring = Tile<2, 1, 2, 4, 1, 4>;
using Tile128 = Tile<2, 2, 2, 2, 2>;
using Tile192 = Tile<3, 2, 2, 4, 1>;
using Tile256 = Tile<4, 2, 2, 4, 1>;

template <int ACT, bool F32>
hipError_t launch_tiles(LinearParams& p, hipStream_t stream) {
    p.group = 4;
    if (tiles<Tile64>(p) <= 512) return launch_shape<ACT, LinearOut<F32, Tile64>, Tile64>(p, stream);
    const long long n128 = tiles<Tile128>(p);
    if (n128 <= 256) return launch_shape<ACT, LinearOut<F32, Tile128Ring>, Tile128Ring>(p, stream);
    const long long last = n128 % 512, rounds192 = (tiles<Tile192>(p) + 255) / 256, rounds256 = (tiles<Tile256>(p) + 255) / 256;
    const long long cost128 = 100 * (n128 / 512) + (last == 0 ? 0 : (last <= 256 ? 65 : 100)), cost192 = 138 * rounds192;
    const long long cost256 = 176 * rounds256 + (rounds256 > 1 ? 0 : (F32 ? 32000 : 6000) / p.K);
    if constexpr (ACT == ACT_ROWS) {
        if (cost256 < cost128 && cost256 < cost192) {
            p.group = 3;
            return launch_shape<ACT, LinearOut<F32, Tile256>, Tile256>(p, stream);
        }
    }
    if (cost128 <= cost192) return launch_shape<ACT, LinearOut<F32, Tile128>, Tile128>(p, stream);
    p.group = 3;
    return launch_shape<ACT, LinearOut<F32, Tile192>, Tile192>(p, stream);
}

template <bool F32, class T>
hipError_t launch_any(LinearParams& p, hipStream_t stream) {
    p.group = 4;
    p.nft = (p.N + T::TF - 1) / T::TF;
    const long long ntt = ((long long)p.M + T::TT - 1) / T::TT, nb = ntt * p.nft;
    if (nb > 0x7FFFFFFFLL) return hipErrorInvalidValue;
    p.ntt = (int)ntt;
    p.nblocks = (int)nb;
    const int grid = (int)(nb < 256 * T::WGS ? nb : 256 * T::WGS);
    hipLaunchKernelGGL((linear_any_kernel<F32, T>), dim3(grid), dim3(T::NT), 0, stream, p);
    return hipGetLastError();
}

template <bool F32, int TB>
hipError_t launch_few(LinearParams& p, hipStream_t stream) {
    hipLaunchKernelGGL((linear_few_kernel<F32, TB>), dim3((p.N + 15) / 16, (p.M + 16 * TB - 1) / (16 * TB)), dim3(512), 0, stream, p);
    return hipGetLastError();
}

template <bool F32>
hipError_t launch(LinearParams& p, hipStream_t stream) {
    fast_divisor(p.L, p.lmul, p.lshift);
    fast_divisor(p.d, p.dmul, p.dshift);
    // Few tokens: a workgroup per 16 features reads every token, so not beyond a
    // workgroup per CU but for very few (us, against the next kernel: 2 tokens x
    // 4608 -> 1152 8.3 and 15.3; 16 x 1152 -> 2304 5.1, 6.4; 32 x 1152 -> 2304 6.1,
    // 6.7; 32 x 4608 -> 1152 15.0, 14.5; 2 x 1152 -> 6912 6.4, 6.6; 8 x 1152 -> 6912 7.0, 6.6).
    const bool aligned = p.K % 8 == 0, narrow = !aligned || p.N <= 16 * 256;
    if (p.M <= 4 || (narrow && p.M <= 16)) return launch_few<F32, 1>(p, stream);
    // Few outputs of more tokens, up to a workgroup per CU whose reads (32 rows of
    // K) the next kernels' longer chains outlast (us, this and the next: 602 x 1152
    // -> 32 4.9, 6.3; 1024 x 1152 -> 64 5.2, 6.5; beyond it 256 x 1152 -> 512 6.9,
    // 6.6; 64 x 4608 -> 1152 18.6, 16.0; 285 x 2017 -> 17 12.3, 26.0).
    const long long blocks = (long long)((p.N + 15) / 16) * ((p.M + 15) / 16);
    if (blocks <= 256 && (!aligned || blocks * p.K <= 256 * 2304)) return launch_few<F32, 1>(p, stream);
    if (narrow && p.M <= 32 && (!aligned || p.K <= 2304)) return launch_few<F32, 2>(p, stream);
    // 64 x 1001 -> 1153 9.0 us against 16.1, 200 tokens 15.0 and 16.6, 9436 x 2062 -> 16 20.1 and 33.1
    if (!aligned && (long long)((p.N + 15) / 16) * ((p.M + 31) / 32) <= 512) return launch_few<F32, 2>(p, stream);
    const bool tail = p.K % (2 * GK) != 0;
    if (p.H > 1) return tail ? launch_tiles<ACT_HEADS_TAIL, F32>(p, stream) : launch_tiles<ACT_HEADS, F32>(p, stream);
    if (aligned) return tail ? launch_tiles<ACT_ROWS_TAIL, F32>(p, stream) : launch_tiles<ACT_ROWS, F32>(p, stream);
    // 64 x 64 tiles against 128 x 128, 1001 -> 1153, us: 200 tokens 16.6 and 26.0, 1000 17.0 and 25.3, 2000 30.7 and
    // 26.0, 8194 87 and 57
    if (tiles<Tile128>(p) <= 128) return launch_any<F32, Tile<1, 1, 2, 2, 2>>(p, stream);
    return launch_any<F32, Tile128>(p, stream);
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
