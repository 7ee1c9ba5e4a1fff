// Internal interface between the host library (argument checks, dispatch,
// plan generator) and the HIP kernels.  Not part of the public ABI.
#ifndef DFA_INTERNAL_H
#define DFA_INTERNAL_H

#include <stddef.h>
#include <hip/hip_runtime_api.h>

namespace dfa {

// One attention launch over B batch entries.  Every destination in dst[]
// receives the same output at the same element offset.
struct AttnLaunch {
    const void* Q;
    const void* K;
    const void* V;
    const void* Rin;   // window kernel: fp32 residual added to the output (may be null)
    void* Rout;        // refresh kernel: fp32 residual output
    void* dst[4];
    int ndst;
    int nout;          // the first nout of dst[] are O, which a caller's next launch reads; the others its output cache
    int B, H, L, d, w;
    int Bcall;         // batch of the whole call (B, or twice it when the launch is its conditional half)
};

// One projection launch of the attention module over B * L tokens.
//   QKV projection: act = X [B][L][H*d], W [3*H*d][H*d], dst[0..2] = Q, K, V
//   output projection: act = O [B][H][L][d], W [H*d][H*d], dst[0..ndst) = copies of Y [B][L][H*d]
struct ProjLaunch {
    const void* W;
    const void* act;
    const void* bias;   // fp32, may be null
    void* dst[4];
    int ndst;
    int B, H, L, d;
};

// Rows of C fp32 values, one per batch entry `stride` elements apart (0: one
// for all); p may be null.
struct Rows {
    const float* p;
    long long stride;
};

// One layer norm launch over B * L tokens; x_f32: X (and dX) are fp32, else bf16.
struct NormLaunch {
    const void* X;
    Rows weight, bias;
    float offset, eps;
    void* Y;
    float* mean;
    float* rstd;
    bool x_f32;
    int B, L, C;
};
struct NormGradLaunch {
    const void* dY;
    const void* X;
    Rows weight;
    float offset;
    const float* mean;
    const float* rstd;
    void* dX;
    float* dweight;
    float* dbias;
    float* partial;    // norm_grad_partials() values
    bool x_f32;
    int B, L, C, groups;
};
constexpr int NORM_C_MAX = 16384;
constexpr int NORM_GROUPS_MAX = 1 << 21;   // a workgroup of up to 1024 lanes each at least
hipError_t launch_layer_norm(const NormLaunch& a, hipStream_t stream);
hipError_t launch_layer_norm_backward(const NormGradLaunch& a, hipStream_t stream);
// fp32 values of workspace that the weight's and the bias's gradients take.
size_t norm_grad_partials(int B, int L, int C, int groups);

// One linear layer; act is a DFA_ACT_ code, y_f32: residual and Y are fp32, else bf16.
struct LinearLaunch {
    const void* X;
    const void* W;
    const float* bias;
    Rows gate;
    const void* residual;
    void* Y;
    int act;
    bool y_f32;
    int B, L, H, K, N;
};
hipError_t launch_linear(const LinearLaunch& a, hipStream_t stream);

// One rotation of Q and K.
constexpr int ROPE_D_MAX = 256, ROPE_AXES_MAX = 4;
struct RopeLaunch {
    const void* Q;
    const void* K;
    void* Qout;
    void* Kout;
    const float* pos;
    long long pos_stride;
    int sections[ROPE_AXES_MAX];
    int naxes;
    double base;
    bool interleaved, inverse;
    int B, Hq, Hk, L, d;
};
hipError_t launch_rope(const RopeLaunch& a, hipStream_t stream);

hipError_t launch_mrae(const void* a, const void* b, size_t n, float eps, double* partial, int max_partials,
                       double* out, hipStream_t stream);
// Workgroups (partial sums) of one MRAE reduction of n elements.
size_t mrae_workgroups(size_t n, int max_partials);
// Partial sums the allocation-free MRAE entry point keeps in device memory of
// its own (a file-scope array of dfa_reduce.hip, one per device).
constexpr int MRAE_SCRATCH_PARTIALS = 1024;
// Device address of that array on the current device (looked up once per device).
hipError_t scratch_partials(double** ptr);
hipError_t launch_add_bf16(const void* a, const void* b, void* out, size_t n, hipStream_t stream);

// Records the message returned by dfa_last_error() for a non-OK status.
int set_error(int status, const char* fmt, ...);

bool head_dim_supported(int d);
bool proj_shape_supported(int H, int d);
hipError_t launch_qkv_proj(const ProjLaunch& a, hipStream_t stream);
hipError_t launch_out_proj(const ProjLaunch& a, hipStream_t stream);
hipError_t launch_full(const AttnLaunch& a, hipStream_t stream);
hipError_t launch_asc(const AttnLaunch& a, hipStream_t stream);  // full attention, separate kernel name
hipError_t launch_refresh(const AttnLaunch& a, hipStream_t stream);
hipError_t launch_window(const AttnLaunch& a, hipStream_t stream);
hipError_t launch_copy(const void* src, void* dst, size_t bytes, hipStream_t stream);

// One-wavefront-per-sequence kernels for L <= SHORT_L_MAX (dfa_short.hip).
constexpr int SHORT_L_MAX = 32;
hipError_t launch_short_full(const AttnLaunch& a, hipStream_t stream);
hipError_t launch_short_asc(const AttnLaunch& a, hipStream_t stream);
hipError_t launch_short_refresh(const AttnLaunch& a, hipStream_t stream);
hipError_t launch_short_window(const AttnLaunch& a, hipStream_t stream);

// The attention operations: short sequences take the per-sequence kernels,
// longer ones the tiled kernels.
inline hipError_t attn_full(const AttnLaunch& a, hipStream_t s) {
    return a.L <= SHORT_L_MAX ? launch_short_full(a, s) : launch_full(a, s);
}
inline hipError_t attn_asc(const AttnLaunch& a, hipStream_t s) {
    return a.L <= SHORT_L_MAX ? launch_short_asc(a, s) : launch_asc(a, s);
}
inline hipError_t attn_refresh(const AttnLaunch& a, hipStream_t s) {
    return a.L <= SHORT_L_MAX ? launch_short_refresh(a, s) : launch_refresh(a, s);
}
inline hipError_t attn_window(const AttnLaunch& a, hipStream_t s) {
    return a.L <= SHORT_L_MAX ? launch_short_window(a, s) : launch_window(a, s);
}

}  // namespace dfa

#endif
