// Projections of the attention module for gfx950 (CDNA4): the fused QKV
// projection in front of the attention path and the output projection behind
// it (the module whose FLOPs Table 2 counts).
//
// Both are D = W Act^T with bf16 operands and fp32 accumulation:
//   W    [N][K]  weights, [out_features][in_features] (y = x W^T + b)
//   Act  token-major activations, K contiguous per token: X [M][K] for the
//        QKV projection, or the attention output O [B][H][L][d] read as the
//        [M][H * d] matrix of merged heads for the output projection
//   D    [N][M]  one output feature per row, one token per column
// The QKV projection's epilogue scatters chunks of eight features straight
// into Q, K or V in the [B][H][L][d] layout of the attention kernels (feature
// f = which * C + head * d + dim, and d is a multiple of 8, so a chunk never
// straddles a head); the output projection stores token-major Y [M][N] to
// every destination given (the unconditional half of an ASC step is one of
// them).
//
// The kernels, their tiles and main loops are in dfa_tiles.h.
//
// What bounds it, at 32768 tokens x 1152 features (PixArt-Sigma at 2048 px):
// in a steady stream of launches the chip's power limit (the shader clock
// falls with N(0, 1) data, where zeros, same instructions, keep it), then the
// output stores and the copies' latency at each k-tile's barrier; LDS bank
// conflicts take 1% of the cycles.  Measured there, against the
// kernels this replaced (whose partial vmcnt wait the barrier's own fence
// undid, and whose epilogue waited for each of its 32 bias loads in turn):
// QKV projection 337 -> 277 us, output projection 133 -> 108 us; at 2048
// tokens 26.2 -> 20.3 and 18.3 -> 13.0 us.
#include "dfa_tiles.h"

namespace dfa {
namespace {

enum { OUT_QKV = 0, OUT_ROWS = 1 };     // epilogue: scatter to Q/K/V, or [M][N] rows

struct GemmParams : Operands {
    uint16_t* dst[4];        // OUT_QKV: Q, K, V; OUT_ROWS: copies of Y
    int ndst;
};

// Output of one wavefront: its blocks of 32 features x 32 tokens, rounded to
// bf16, pass one by one through the wavefront's scratch as [token][feature]
// rows (chunk c of row t at c ^ ((t >> 2) & 3)), so that they leave as 16-byte
// chunks in row order.  A lane holds four consecutive features of a token and
// lane + 32 the next four: one exchange gives each lane a whole chunk.
template <int OUT, class T, bool WHOLE>
__device__ __forceinline__ void store_tile(const GemmParams& p, f32x16 (&acc)[T::MB][T::NB], uint16_t* scratch, int nw0,
                                           int tw0, int lane) {
    // opaque: nothing of the epilogue's addressing is to be kept in registers
    // through the next tile's k loop
    asm volatile("" : "+v"(lane));
    const int r32 = lane & 31, h = lane >> 5, srow = lane >> 2, sc = lane & 3;
    const int C = p.K;                                                    // OUT_QKV: N = 3 K
    const uint16_t* from = scratch + srow * 32 + ((sc ^ (srow >> 2)) << 3);   // and row srow + 16: same swizzle
    size_t trow[T::NB][2];
#pragma unroll
    for (int nb = 0; nb < T::NB; ++nb)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int t = tw0 + 32 * nb + 16 * i + srow;
            // OUT_QKV: (b H + head) L + l rows of d, with l = t - b L
            if constexpr (OUT == OUT_QKV)
                trow[nb][i] = ((size_t)t + (size_t)fast_div(min(t, p.M - 1), p.lmul, p.lshift) * (p.H - 1) * p.L) * p.d;
            else
                trow[nb][i] = (size_t)t * p.N;
        }
#pragma unroll
    for (int mb = 0; mb < T::MB; ++mb) {
        const int f = nw0 + 32 * mb + 8 * sc;
        uint16_t* out;
        if constexpr (OUT == OUT_QKV) {
            const int which = f >= 2 * C ? 2 : (f >= C ? 1 : 0), fr = f - which * C;
            const int head = fast_div(fr, p.dmul, p.dshift);
            out = (which == 2 ? p.dst[2] : (which == 1 ? p.dst[1] : p.dst[0])) + (size_t)head * (p.L - 1) * p.d + fr;
        } else {
            out = p.dst[0] + f;
        }
#pragma unroll
        for (int nb = 0; nb < T::NB; ++nb) {
            const f32x16& a = acc[mb][nb];
#pragma unroll
            for (int jp = 0; jp < 2; ++jp) {
                uint32_t x0 = pack_bf16x2(a[8 * jp], a[8 * jp + 1]), x1 = pack_bf16x2(a[8 * jp + 2], a[8 * jp + 3]);
                uint32_t y0 = pack_bf16x2(a[8 * jp + 4], a[8 * jp + 5]), y1 = pack_bf16x2(a[8 * jp + 6], a[8 * jp + 7]);
                xchg32(x0, y0);
                xchg32(x1, y1);
                *(u32x4*)(scratch + r32 * 32 + (((2 * jp + h) ^ ((r32 >> 2) & 3)) << 3)) = u32x4{x0, x1, y0, y1};
            }
            __builtin_amdgcn_wave_barrier();   // the wavefront's LDS accesses complete in order
            u32x4 val[2] = {*(const u32x4*)from, *(const u32x4*)(from + 16 * 32)};
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int t = tw0 + 32 * nb + 16 * i + srow;
                if (!WHOLE && (t >= p.M || f >= p.N)) continue;
                *(u32x4*)(out + trow[nb][i]) = val[i];
                if constexpr (OUT == OUT_ROWS)
                    for (int di = 1; di < p.ndst; ++di) *(u32x4*)(p.dst[di] + f + trow[nb][i]) = val[i];
            }
        }
    }
}

template <int WHICH, class T>
struct Output {
    using Params = GemmParams;
    static constexpr int SCRATCH = 32 * 32;   // one 32 x 32 block of output, or the biases
    static constexpr bool FROM_BIAS = true;
    static_assert(8 * T::MB <= 64 && 64 * T::MB <= SCRATCH, "biases of a wavefront");
    __device__ __forceinline__ void ahead(const GemmParams&, int, int, int, bool) {}
    template <bool WHOLE>
    __device__ __forceinline__ void store(const GemmParams& p, f32x16 (&acc)[T::MB][T::NB], uint16_t* scratch, int nw0, int tw0,
                                          int lane) {
        store_tile<WHICH, T, WHOLE>(p, acc, scratch, nw0, tw0, lane);
    }
};

// Tile shapes, features x tokens, and the rule between them (all measured at
// 16 heads x 72 and other widths from 384 to 2304 features, times in us):
//   64 x 64, ring      while one such tile per CU covers the output (600 tokens
//                      x 1152 features 7.3 against 12.6 for the next shape;
//                      at 528 tiles 18.6 against 15.6)
//   128 x 128, ring    the same (2048 tokens x 1152: 13.0 against 16.4 for the
//                      next; at 288 tiles 25.6 against 18.6)
//   128 x 128, stream  two workgroups per CU, or
//   192 x 256, stream  one: by the rounds that each needs.  A round of the
//                      larger tile takes 1.25 of the smaller's (24 against 19
//                      at K = 1152) for 1.5 of its output; a last round of the
//                      smaller with one workgroup on a CU takes 0.65.
// Block order: a weight that fits one XCD's 4 MB L2 stays there while an XCD
// walks all feature tiles of one token tile after another.  A larger one (the
// QKV projection's 7.6 MB at C = 1152) would be fetched again for every token
// tile, so the tiles go in groups of 8 token tiles, feature tile by feature
// tile: an XCD's resident workgroups then share both operands' tiles.
using Tile64 = Tile<1, 1, 2, 2, 2, 4>;
using Tile128Ring = Tile<2, 1, 2, 4, 1, 4>;
using Tile128 = Tile<2, 2, 2, 2, 2>;
using Tile192 = Tile<3, 2, 2, 4, 1>;

template <int ACT, int OUT>
hipError_t launch_gemm(GemmParams& p, hipStream_t stream) {
    p.group = (long long)p.N * p.K * 2 > (4LL << 20) ? 8 : 1;
    if (tiles<Tile64>(p) <= 256) return launch_shape<ACT, Output<OUT, Tile64>, Tile64>(p, stream);
    const long long n128 = tiles<Tile128>(p), n192 = tiles<Tile192>(p);
    if (n128 <= 256) return launch_shape<ACT, Output<OUT, Tile128Ring>, Tile128Ring>(p, stream);
    const long long last = n128 % 512;
    const long long rounds128 = 100 * (n128 / 512) + (last == 0 ? 0 : (last <= 256 ? 65 : 100));
    const long long rounds192 = 125 * ((n192 + 255) / 256);
    if (rounds192 < rounds128) return launch_shape<ACT, Output<OUT, Tile192>, Tile192>(p, stream);
    return launch_shape<ACT, Output<OUT, Tile128>, Tile128>(p, stream);
}

}  // namespace

bool proj_shape_supported(int H, int d) { return H > 0 && (d == 64 || d == 72) && (H * d) % 128 == 0; }

hipError_t launch_qkv_proj(const ProjLaunch& a, hipStream_t stream) {
    GemmParams p{};
    p.W = (const uint16_t*)a.W;
    p.act = (const uint16_t*)a.act;
    p.bias = (const float*)a.bias;
    for (int i = 0; i < 3; ++i) p.dst[i] = (uint16_t*)a.dst[i];
    p.ndst = 3;
    p.L = a.L;
    p.H = a.H;
    p.d = a.d;
    p.M = a.B * a.L;
    p.K = a.H * a.d;
    p.N = 3 * p.K;
    return launch_gemm<ACT_ROWS, OUT_QKV>(p, stream);
}

hipError_t launch_out_proj(const ProjLaunch& a, hipStream_t stream) {
    GemmParams p{};
    p.W = (const uint16_t*)a.W;
    p.act = (const uint16_t*)a.act;
    p.bias = (const float*)a.bias;
    p.ndst = a.ndst;
    for (int i = 0; i < 4; ++i) p.dst[i] = (uint16_t*)(i < a.ndst ? a.dst[i] : nullptr);
    p.L = a.L;
    p.H = a.H;
    p.d = a.d;
    p.M = a.B * a.L;
    p.K = a.H * a.d;
    p.N = p.K;
    return launch_gemm<ACT_HEADS, OUT_ROWS>(p, stream);
}

}  // namespace dfa
