// C entry points of the encoder (include/lccrf_encoder.h): argument checks, then launches.  No allocation, no
// synchronisation, nothing that throws.
#include "../../include/lccrf_encoder.h"
#include "lccrf_encoder.h"

using namespace lccrf::enc;

namespace {

inline bool type_ok(int dt) { return dt == LCCRF_F32 || dt == LCCRF_BF16; }
inline size_t size_of(int dt) { return dt == LCCRF_F32 ? 4 : 2; }
inline bool lies(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline AnyRows rows(const lccrf_rows& r) { return {r.data, r.batch, r.row}; }
inline bool positions_ok(int B, int N, int D) { return B >= 1 && N >= 1 && D >= 1 && static_cast<int64_t>(B) * N <= kMaxPositions; }
inline bool conv_ok(int B, int N, int D, int K) { return positions_ok(B, N, D) && K >= LCCRF_MIN_TAPS && K <= LCCRF_MAX_TAPS; }
inline bool scan_ok(int B, int N, int D, int S, int G) {
    return positions_ok(B, N, D) && D <= 1 << 22 && S >= 1 && S <= LCCRF_MAX_STATES && G >= 1 && G <= D && D % G == 0 && static_cast<int64_t>(G) * S < (1 << 27);
}
inline bool embed_grad_ok(int64_t n, int V, int D) { return n >= 0 && n <= (int64_t{1} << 30) && V >= 1 && V <= 1 << 30 && D >= 1; }

inline int status(hipError_t e) { return e == hipSuccess ? LCCRF_OK : e == hipErrorInvalidValue ? LCCRF_EINVAL : LCCRF_ELAUNCH; }

inline int scan_inputs(const lccrf_scan_inputs* in, int dtype) {
    if (!in || !in->x.data || !in->dt.data || !in->Bm.data || !in->Cm.data || !in->A) return LCCRF_ENULL;
    const size_t e = size_of(dtype);
    if (!lies(in->x.data, e) || !lies(in->dt.data, e) || !lies(in->Bm.data, e) || !lies(in->Cm.data, e) || !lies(in->z.data, e) || !lies(in->A, 4) ||
        !lies(in->D, 4) || !lies(in->dt_bias, 4))
        return LCCRF_EALIGN;
    return LCCRF_OK;
}
inline ScanIn scan_in(const lccrf_scan_inputs* in, const int32_t* lengths, int B, int N, int D, int S, int G) {
    return {rows(in->x), rows(in->dt), rows(in->Bm), rows(in->Cm), rows(in->z), in->b_group, in->c_group, in->A, in->D, in->dt_bias, lengths, B, N, D, S, G};
}

}  // namespace

extern "C" {

int lccrf_embed(const void* table, lccrf_dtype dt, int V, int D, int64_t table_row, const int32_t* ids, int64_t n, float scale, void* out, void* stream) {
    if (!type_ok(dt) || V < 1 || D < 1 || n < 0) return LCCRF_EINVAL;
    if (n == 0) return LCCRF_OK;
    if (!table || !ids || !out) return LCCRF_ENULL;
    if (!lies(table, size_of(dt)) || !lies(ids, 4) || !lies(out, size_of(dt))) return LCCRF_EALIGN;
    return status(launch_embed(dt, table, V, D, table_row, ids, n, scale, out, static_cast<hipStream_t>(stream)));
}

size_t lccrf_embed_grad_workspace_bytes(int64_t n, int V, int D) { return embed_grad_ok(n, V, D) ? embed_grad_workspace(n, V, D) : 0; }

int lccrf_embed_grad(const lccrf_rows* dout, lccrf_dtype dt, const int32_t* ids, int B, int N, int V, int D, float scale, void* grad, void* workspace,
                     size_t workspace_bytes, void* stream) {
    if (!type_ok(dt) || B < 0 || N < 0 || !embed_grad_ok(static_cast<int64_t>(B) * N, V, D)) return LCCRF_EINVAL;
    const int64_t n = static_cast<int64_t>(B) * N;
    if (!grad || (n > 0 && (!dout || !dout->data || !ids))) return LCCRF_ENULL;
    if (!workspace || workspace_bytes < embed_grad_workspace(n, V, D)) return LCCRF_EWORKSPACE;
    if (!lies(grad, size_of(dt)) || !lies(ids, 4) || !lies(workspace, 256) || (n > 0 && !lies(dout->data, size_of(dt)))) return LCCRF_EALIGN;
    const AnyRows d = n > 0 ? rows(*dout) : AnyRows{};
    return status(launch_embed_grad(dt, d, ids, B, N, V, D, scale, grad, workspace, static_cast<hipStream_t>(stream)));
}

int lccrf_conv(const lccrf_rows* x, lccrf_dtype dt, const float* weight, const float* bias, const void* state, const int32_t* lengths, int B, int N, int D,
               int K, void* out, void* final_state, void* stream) {
    if (!type_ok(dt) || !conv_ok(B, N, D, K)) return LCCRF_EINVAL;
    if (!x || !x->data || !weight || !out) return LCCRF_ENULL;
    const size_t e = size_of(dt);
    if (!lies(x->data, e) || !lies(weight, 4) || !lies(bias, 4) || !lies(state, e) || !lies(lengths, 4) || !lies(out, e) || !lies(final_state, e)) return LCCRF_EALIGN;
    if (state && state == final_state) return LCCRF_EINVAL;  // other threads still read the one while the other is written
    return status(launch_conv(dt, rows(*x), weight, bias, state, lengths, B, N, D, K, out, final_state, static_cast<hipStream_t>(stream)));
}

size_t lccrf_conv_grad_workspace_bytes(int B, int N, int D, int K) { return conv_ok(B, N, D, K) ? conv_grad_workspace(B, N, D, K) : 0; }

int lccrf_conv_grad(const lccrf_rows* dout, const lccrf_rows* x, lccrf_dtype dt, const float* weight, const float* bias, const void* state,
                    const int32_t* lengths, int B, int N, int D, int K, void* dx, float* dweight, float* dbias, void* dstate, void* workspace,
                    size_t workspace_bytes, void* stream) {
    if (!type_ok(dt) || !conv_ok(B, N, D, K) || (dstate && !state)) return LCCRF_EINVAL;
    if (!dout || !dout->data || !x || !x->data || !weight || !dx || !dweight) return LCCRF_ENULL;
    if (!workspace || workspace_bytes < conv_grad_workspace(B, N, D, K)) return LCCRF_EWORKSPACE;
    const size_t e = size_of(dt);
    if (!lies(dout->data, e) || !lies(x->data, e) || !lies(weight, 4) || !lies(bias, 4) || !lies(state, e) || !lies(lengths, 4) || !lies(dx, e) || !lies(dweight, 4) ||
        !lies(dbias, 4) || !lies(dstate, e) || !lies(workspace, 256))
        return LCCRF_EALIGN;
    return status(launch_conv_grad(dt, rows(*dout), rows(*x), weight, bias, state, lengths, B, N, D, K, dx, dweight, dbias, dstate, workspace,
                                   static_cast<hipStream_t>(stream)));
}

int lccrf_conv_step(const void* x, int64_t x_row, lccrf_dtype dt, const float* weight, const float* bias, void* state, int B, int D, int K, void* out,
                    void* stream) {
    if (!type_ok(dt) || !conv_ok(B, 1, D, K)) return LCCRF_EINVAL;
    if (!x || !weight || !state || !out) return LCCRF_ENULL;
    const size_t e = size_of(dt);
    if (!lies(x, e) || !lies(weight, 4) || !lies(bias, 4) || !lies(state, e) || !lies(out, e)) return LCCRF_EALIGN;
    return status(launch_conv_step(dt, x, x_row, weight, bias, state, B, D, K, out, static_cast<hipStream_t>(stream)));
}

size_t lccrf_state_scan_saved_bytes(int B, int N, int D, int S) { return scan_ok(B, N, D, S, 1) ? scan_saved_bytes(B, N, D, S) : 0; }
size_t lccrf_state_scan_workspace_bytes(int B, int N, int D, int S, int G) { return scan_ok(B, N, D, S, G) ? scan_workspace(B, N, D, S, G) : 0; }
size_t lccrf_state_scan_grad_workspace_bytes(int B, int N, int D, int S, int G, int with_saved) {
    return scan_ok(B, N, D, S, G) ? scan_grad_workspace(B, N, D, S, G, with_saved != 0) : 0;
}

int lccrf_state_scan(const lccrf_scan_inputs* in, lccrf_dtype dtype, const int32_t* lengths, int B, int N, int D, int S, int G, const float* state, void* out,
                     float* final_state, void* saved, void* workspace, size_t workspace_bytes, void* stream) {
    if (!type_ok(dtype) || !scan_ok(B, N, D, S, G)) return LCCRF_EINVAL;
    if (!out) return LCCRF_ENULL;
    if (const int rc = scan_inputs(in, dtype)) return rc;
    if (!workspace || workspace_bytes < scan_workspace(B, N, D, S, G)) return LCCRF_EWORKSPACE;
    if (!lies(lengths, 4) || !lies(state, 4) || !lies(out, size_of(dtype)) || !lies(final_state, 4) || !lies(saved, 256) || !lies(workspace, 256)) return LCCRF_EALIGN;
    return status(launch_state_scan(dtype, scan_in(in, lengths, B, N, D, S, G), state, out, final_state, saved, workspace, static_cast<hipStream_t>(stream)));
}

int lccrf_state_scan_grad(const lccrf_rows* dout, const lccrf_scan_inputs* in, lccrf_dtype dtype, const int32_t* lengths, int B, int N, int D, int S, int G,
                          const float* state, const void* saved, const lccrf_scan_grads* g, void* workspace, size_t workspace_bytes, void* stream) {
    if (!type_ok(dtype) || !scan_ok(B, N, D, S, G)) return LCCRF_EINVAL;
    if (!dout || !dout->data || !g || !g->dx || !g->ddt || !g->dBm || !g->dCm || !g->dA) return LCCRF_ENULL;
    if (const int rc = scan_inputs(in, dtype)) return rc;
    if ((in->z.data != nullptr) != (g->dz != nullptr) || (g->dstate && !state)) return LCCRF_EINVAL;
    if (!workspace || workspace_bytes < scan_grad_workspace(B, N, D, S, G, saved != nullptr)) return LCCRF_EWORKSPACE;
    const size_t e = size_of(dtype);
    if (!lies(dout->data, e) || !lies(lengths, 4) || !lies(state, 4) || !lies(saved, 256) || !lies(workspace, 256) || !lies(g->dx, e) || !lies(g->ddt, e) || !lies(g->dBm, e) ||
        !lies(g->dCm, e) || !lies(g->dz, e) || !lies(g->dA, 4) || !lies(g->dD, 4) || !lies(g->ddt_bias, 4) || !lies(g->dstate, 4))
        return LCCRF_EALIGN;
    const ScanGrads grads{g->dx, g->ddt, g->dBm, g->dCm, g->dz, g->dA, g->dD, g->ddt_bias, g->dstate};
    return status(launch_state_scan_grad(dtype, rows(*dout), scan_in(in, lengths, B, N, D, S, G), state, saved, grads, workspace, static_cast<hipStream_t>(stream)));
}

int lccrf_state_step(const lccrf_scan_inputs* in, lccrf_dtype dtype, int B, int D, int S, int G, float* state, void* out, void* stream) {
    if (!type_ok(dtype) || !scan_ok(B, 1, D, S, G)) return LCCRF_EINVAL;
    if (!state || !out) return LCCRF_ENULL;
    if (const int rc = scan_inputs(in, dtype)) return rc;
    if (!lies(state, 4) || !lies(out, size_of(dtype))) return LCCRF_EALIGN;
    return status(launch_state_step(dtype, scan_in(in, nullptr, B, 1, D, S, G), state, out, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
