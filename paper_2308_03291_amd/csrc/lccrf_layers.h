// Shared by the kernels behind include/lccrf_layers.h (gated recurrence, group norm, distillation): argument blocks and launch entry points.
#pragma once

#include "lccrf_encoder.h"

namespace lccrf {
namespace enc {

struct RecurIn {
    AnyRows x, f, g, z;
    const float *decay, *f_bias, *g_bias;
    float rate;
    const int32_t* lengths;
    int B, N, D;
};
struct RecurGrads {
    void *dx, *df, *dg, *dz;
    float *ddecay, *df_bias, *dg_bias, *dstate;
};

// dtype 0: float, 1: bfloat16.  All return the status of their launches.
size_t recur_saved_bytes(int B, int N, int D);
size_t recur_workspace(int B, int N, int D);
size_t recur_grad_workspace(int B, int N, int D, bool with_saved);
hipError_t launch_recur(int dtype, const RecurIn& in, const float* state, void* out, float* final_state, float* saved, void* ws, hipStream_t st);
hipError_t launch_recur_grad(int dtype, AnyRows dout, const RecurIn& in, const float* state, const float* saved, const RecurGrads& g, void* ws, hipStream_t st);
hipError_t launch_recur_step(int dtype, const RecurIn& in, float* state, void* out, hipStream_t st);

struct NormIn {
    AnyRows x;
    const float *weight, *bias;
    const int32_t* lengths;
    int B, N, D, G;
    float eps;
    bool silu, alone;  // alone: every position by itself
};
size_t norm_workspace(int dtype, int B, int N, int D, int G, bool alone);
size_t norm_grad_workspace(int dtype, int B, int N, int D, int G, bool alone);
hipError_t launch_norm(int dtype, const NormIn& in, void* out, float* stats, void* ws, hipStream_t st);
hipError_t launch_norm_grad(int dtype, AnyRows dout, const NormIn& in, const float* stats, void* dx, float* dweight, float* dbias, void* ws, hipStream_t st);

struct DistillIn {
    const void* logits;
    int64_t row;
    const int32_t* ids;
    const float* teacher;
    int64_t n;
    int V, K;
    float temperature;
};
hipError_t launch_distill(int dtype, const DistillIn& in, float* loss, float* lse, hipStream_t st);
hipError_t launch_distill_grad(int dtype, const float* dloss, const DistillIn& in, const float* lse, float* loss, void* dlogits, hipStream_t st);

__device__ __forceinline__ int length_at(const int32_t* lengths, int b, int N) {
    if (!lengths) return N;
    const int n = lengths[b];
    return n < 0 ? 0 : n > N ? N : n;
}

// A barrier for what goes through LDS alone: loads and stores of global memory stay in flight across it.
__device__ __forceinline__ void lds_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Over `team` neighbouring lanes, a power of two up to 64, the same in all of them: f of a lane's and the other half's, from neighbours on.  In registers
// throughout: permutations of four lanes, mirrored halves and rows of sixteen, swapped rows and halves.
template <int CTRL> __device__ __forceinline__ float moved(float x) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}
template <typename F> __device__ __forceinline__ float across(float v, int team, F f) {
    if (team > 1) v = f(v, moved<0xB1>(v));
    if (team > 2) v = f(v, moved<0x4E>(v));
    if (team > 4) v = f(v, moved<0x141>(v));
    if (team > 8) v = f(v, moved<0x140>(v));
    if (team > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    if (team > 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return v;
}
__device__ __forceinline__ float sum_across(float v, int team) {
    return across(v, team, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float max_across(float v, int team) {
    return across(v, team, [](float a, float b) { return __builtin_elementwise_maximum(a, b); });
}

}  // namespace enc
}  // namespace lccrf
