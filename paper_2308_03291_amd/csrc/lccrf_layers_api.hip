// C entry points of include/lccrf_layers.h: argument checks, then launches.  No allocation, no synchronisation, nothing that throws.
#include "../../include/lccrf_layers.h"
#include "lccrf_layers.h"

using namespace lccrf::enc;

namespace {

inline bool type_ok(int dt) { return dt == LCCRF_F32 || dt == LCCRF_BF16; }
inline size_t size_of(int dt) { return dt == LCCRF_F32 ? 4 : 2; }
inline bool lies(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline AnyRows rows(const lccrf_rows& r) { return {r.data, r.batch, r.row}; }
inline bool positive(float v) { return v > 0.0f && v <= 3.402823466e38f; }
// A scalar that kernels divide by, or take a root's inverse of: below the least normal float that is none.
inline bool normal(float v) { return positive(v) && v >= 1.17549435e-38f; }
inline bool sizes_ok(int B, int N, int D) { return B >= 1 && N >= 1 && D >= 1 && D <= 1 << 22 && static_cast<int64_t>(B) * N <= kMaxPositions; }
inline bool norm_ok(int dt, int B, int N, int D, int G) { return type_ok(dt) && sizes_ok(B, N, D) && G >= 1 && G <= D && D % G == 0; }
inline bool distill_ok(int dt, int64_t n, int V, int K, float t) {
    return type_ok(dt) && n >= 0 && n < (int64_t{1} << 31) && V >= 1 && V <= 1 << 30 && K >= 1 && K <= LCCRF_MAX_TOP && normal(t);
}

inline int status(hipError_t e) { return e == hipSuccess ? LCCRF_OK : e == hipErrorInvalidValue ? LCCRF_EINVAL : LCCRF_ELAUNCH; }

inline int recur_inputs(const lccrf_recurrence_inputs* in, int dtype) {
    if (!in || !in->x.data || !in->f.data || !in->g.data || !in->decay) return LCCRF_ENULL;
    const size_t e = size_of(dtype);
    if (!lies(in->x.data, e) || !lies(in->f.data, e) || !lies(in->g.data, e) || !lies(in->z.data, e) || !lies(in->decay, 4) || !lies(in->f_bias, 4) || !lies(in->g_bias, 4))
        return LCCRF_EALIGN;
    return LCCRF_OK;
}
inline RecurIn recur_in(const lccrf_recurrence_inputs* in, float rate, const int32_t* lengths, int B, int N, int D) {
    return {rows(in->x), rows(in->f), rows(in->g), rows(in->z), in->decay, in->f_bias, in->g_bias, rate, lengths, B, N, D};
}

// A size of 0 is that of a call that is not served: what is asked for is 256 bytes more than what is needed.
inline size_t asked(size_t need) { return need + 256; }
inline bool room(const void* workspace, size_t bytes, size_t need) { return need == 0 || (workspace && bytes >= need); }

inline int distill_inputs(const void* logits, int dtype, const int32_t* ids, const float* teacher) {
    if (!logits || !ids || !teacher) return LCCRF_ENULL;
    return lies(logits, size_of(dtype)) && lies(ids, 4) && lies(teacher, 4) ? LCCRF_OK : LCCRF_EALIGN;
}

}  // namespace

extern "C" {

size_t lccrf_recurrence_saved_bytes(int B, int N, int D) { return sizes_ok(B, N, D) ? recur_saved_bytes(B, N, D) : 0; }
size_t lccrf_recurrence_workspace_bytes(int B, int N, int D) { return sizes_ok(B, N, D) ? asked(recur_workspace(B, N, D)) : 0; }
size_t lccrf_recurrence_grad_workspace_bytes(int B, int N, int D, int with_saved) {
    return sizes_ok(B, N, D) ? asked(recur_grad_workspace(B, N, D, with_saved != 0)) : 0;
}

int lccrf_recurrence(const lccrf_recurrence_inputs* in, lccrf_dtype dtype, float rate, const int32_t* lengths, int B, int N, int D, const float* state, void* out,
                     float* final_state, void* saved, void* workspace, size_t workspace_bytes, void* stream) {
    if (!type_ok(dtype) || !sizes_ok(B, N, D) || !positive(rate)) return LCCRF_EINVAL;
    if (!out) return LCCRF_ENULL;
    if (const int rc = recur_inputs(in, dtype)) return rc;
    if (!room(workspace, workspace_bytes, recur_workspace(B, N, D))) return LCCRF_EWORKSPACE;
    if (!lies(lengths, 4) || !lies(state, 4) || !lies(out, size_of(dtype)) || !lies(final_state, 4) || !lies(saved, 256) || !lies(workspace, 256)) return LCCRF_EALIGN;
    return status(launch_recur(dtype, recur_in(in, rate, lengths, B, N, D), state, out, final_state, static_cast<float*>(saved), workspace, static_cast<hipStream_t>(stream)));
}

int lccrf_recurrence_grad(const lccrf_rows* dout, const lccrf_recurrence_inputs* in, lccrf_dtype dtype, float rate, const int32_t* lengths, int B, int N, int D,
                          const float* state, const void* saved, const lccrf_recurrence_grads* g, void* workspace, size_t workspace_bytes, void* stream) {
    if (!type_ok(dtype) || !sizes_ok(B, N, D) || !positive(rate)) return LCCRF_EINVAL;
    if (!dout || !dout->data || !g || !g->dx || !g->df || !g->dg || !g->ddecay) return LCCRF_ENULL;
    if (const int rc = recur_inputs(in, dtype)) return rc;
    if ((in->z.data != nullptr) != (g->dz != nullptr) || (g->dstate && !state)) return LCCRF_EINVAL;
    if (!room(workspace, workspace_bytes, recur_grad_workspace(B, N, D, saved != nullptr))) return LCCRF_EWORKSPACE;
    const size_t e = size_of(dtype);
    if (!lies(dout->data, e) || !lies(lengths, 4) || !lies(state, 4) || !lies(saved, 256) || !lies(workspace, 256) || !lies(g->dx, e) || !lies(g->df, e) || !lies(g->dg, e) ||
        !lies(g->dz, e) || !lies(g->ddecay, 4) || !lies(g->df_bias, 4) || !lies(g->dg_bias, 4) || !lies(g->dstate, 4))
        return LCCRF_EALIGN;
    const RecurGrads grads{g->dx, g->df, g->dg, g->dz, g->ddecay, g->df_bias, g->dg_bias, g->dstate};
    return status(launch_recur_grad(dtype, rows(*dout), recur_in(in, rate, lengths, B, N, D), state, static_cast<const float*>(saved), grads, workspace,
                                    static_cast<hipStream_t>(stream)));
}

int lccrf_recurrence_step(const lccrf_recurrence_inputs* in, lccrf_dtype dtype, float rate, int B, int D, float* state, void* out, void* stream) {
    if (!type_ok(dtype) || !sizes_ok(B, 1, D) || !positive(rate)) return LCCRF_EINVAL;
    if (!state || !out) return LCCRF_ENULL;
    if (const int rc = recur_inputs(in, dtype)) return rc;
    if (!lies(state, 4) || !lies(out, size_of(dtype))) return LCCRF_EALIGN;
    return status(launch_recur_step(dtype, recur_in(in, rate, nullptr, B, 1, D), state, out, static_cast<hipStream_t>(stream)));
}

size_t lccrf_group_norm_workspace_bytes(lccrf_dtype dtype, int B, int N, int D, int G, int per_position) {
    return norm_ok(dtype, B, N, D, G) ? asked(norm_workspace(dtype, B, N, D, G, per_position != 0)) : 0;
}
size_t lccrf_group_norm_grad_workspace_bytes(lccrf_dtype dtype, int B, int N, int D, int G, int per_position) {
    return norm_ok(dtype, B, N, D, G) ? asked(norm_grad_workspace(dtype, B, N, D, G, per_position != 0)) : 0;
}

int lccrf_group_norm(const lccrf_rows* x, lccrf_dtype dtype, const float* weight, const float* bias, const int32_t* lengths, int B, int N, int D, int G, int per_position,
                     float eps, int silu, void* out, float* stats, void* workspace, size_t workspace_bytes, void* stream) {
    if (!norm_ok(dtype, B, N, D, G) || !normal(eps)) return LCCRF_EINVAL;
    if (!x || !x->data || !out) return LCCRF_ENULL;
    if (!room(workspace, workspace_bytes, norm_workspace(dtype, B, N, D, G, per_position != 0))) return LCCRF_EWORKSPACE;
    const size_t e = size_of(dtype);
    if (!lies(x->data, e) || !lies(weight, 4) || !lies(bias, 4) || !lies(lengths, 4) || !lies(out, e) || !lies(stats, 4) || !lies(workspace, 256)) return LCCRF_EALIGN;
    const NormIn in{rows(*x), weight, bias, lengths, B, N, D, G, eps, silu != 0, per_position != 0};
    return status(launch_norm(dtype, in, out, stats, workspace, static_cast<hipStream_t>(stream)));
}

int lccrf_group_norm_grad(const lccrf_rows* dout, const lccrf_rows* x, lccrf_dtype dtype, const float* weight, const float* bias, const int32_t* lengths, int B, int N,
                          int D, int G, int per_position, float eps, int silu, const float* stats, void* dx, float* dweight, float* dbias, void* workspace,
                          size_t workspace_bytes, void* stream) {
    if (!norm_ok(dtype, B, N, D, G) || !normal(eps)) return LCCRF_EINVAL;
    if (!dout || !dout->data || !x || !x->data || !dx) return LCCRF_ENULL;
    if (!room(workspace, workspace_bytes, norm_grad_workspace(dtype, B, N, D, G, per_position != 0))) return LCCRF_EWORKSPACE;
    const size_t e = size_of(dtype);
    if (!lies(dout->data, e) || !lies(x->data, e) || !lies(weight, 4) || !lies(bias, 4) || !lies(lengths, 4) || !lies(stats, 4) || !lies(dx, e) || !lies(dweight, 4) ||
        !lies(dbias, 4) || !lies(workspace, 256))
        return LCCRF_EALIGN;
    const NormIn in{rows(*x), weight, bias, lengths, B, N, D, G, eps, silu != 0, per_position != 0};
    return status(launch_norm_grad(dtype, rows(*dout), in, stats, dx, dweight, dbias, workspace, static_cast<hipStream_t>(stream)));
}

int lccrf_distill(const void* logits, int64_t logits_row, lccrf_dtype dtype, const int32_t* ids, const float* teacher, int64_t n, int V, int K, float temperature,
                  float* loss, float* lse, void* stream) {
    if (!distill_ok(dtype, n, V, K, temperature)) return LCCRF_EINVAL;
    if (n == 0) return LCCRF_OK;
    if (!loss || !lse) return LCCRF_ENULL;
    if (const int rc = distill_inputs(logits, dtype, ids, teacher)) return rc;
    if (!lies(loss, 4) || !lies(lse, 4)) return LCCRF_EALIGN;
    return status(launch_distill(dtype, {logits, logits_row, ids, teacher, n, V, K, temperature}, loss, lse, static_cast<hipStream_t>(stream)));
}

int lccrf_distill_grad(const float* dloss, const void* logits, int64_t logits_row, lccrf_dtype dtype, const int32_t* ids, const float* teacher, int64_t n, int V, int K,
                       float temperature, const float* lse, float* loss, void* dlogits, void* stream) {
    if (!distill_ok(dtype, n, V, K, temperature)) return LCCRF_EINVAL;
    if (n == 0) return LCCRF_OK;
    if (!dloss || !dlogits) return LCCRF_ENULL;
    if (const int rc = distill_inputs(logits, dtype, ids, teacher)) return rc;
    if (!lies(dloss, 4) || !lies(lse, 4) || !lies(loss, 4) || !lies(dlogits, size_of(dtype))) return LCCRF_EALIGN;
    if (logits == dlogits && logits_row != V && n > 1) return LCCRF_EINVAL;
    return status(launch_distill_grad(dtype, dloss, {logits, logits_row, ids, teacher, n, V, K, temperature}, lse, loss, dlogits, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
