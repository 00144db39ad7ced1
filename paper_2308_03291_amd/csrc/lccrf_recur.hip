// Gated linear recurrence: forward pass and single-token form (lccrf_recur.h says how the work is spread).
#include "lccrf_recur.h"

namespace lccrf {
namespace enc {
namespace {

enum { kOut = 1, kSave = 2, kEnds = 4 };

struct RecurRun {
    RecurIn in;
    const float* state;
    void* out;
    float* final_state;
    float* saved;  // [B][ceil(N / kRecurSave)][D]
    float* ends;   // segments > 1: [B][segments][D][2]: what a segment makes of a state, the first one of the call's (kEnds: written)
    RecurPlan plan;
};

template <typename T, int V, int P, int W, int MODE, bool GATED>
__global__ __launch_bounds__(64 * W) void recur_kernel(RecurRun r) {
    typedef float Pair __attribute__((ext_vector_type(2 * V)));
    typedef Pair AnyPair __attribute__((aligned(4)));
    __shared__ Pair pairs[W > 1 ? 2 : 1][W][64];
    const RecurIn& in = r.in;
    const int lane = threadIdx.x & 63, w = W > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const unsigned which = blockIdx.x / r.plan.tiles;
    const int tile = blockIdx.x - which * r.plan.tiles;
    const int b = which / r.plan.segments, seg = which - b * r.plan.segments;
    const Lane<V> my(tile, lane, in.D);
    const unsigned bytes = static_cast<unsigned>(my.c) * sizeof(T);
    const int len = length_at(in.lengths, b, in.N), begin = seg * r.plan.seg_len;
    const int stop = in.N - begin < r.plan.seg_len ? in.N : begin + r.plan.seg_len, end = stop < len ? stop : len;
    T* out = static_cast<T*>(r.out) + static_cast<int64_t>(b) * in.N * in.D;

    RecurChannel ch[V];
    float carry[V], total[V];  // the state before the block; kEnds: what of it is the product of the decays
#pragma unroll
    for (int j = 0; j < V; ++j) {
        ch[j] = recur_channel(in, my.c + j);
        carry[j] = seg == 0 && r.state ? r.state[static_cast<int64_t>(b) * in.D + my.c + j] : 0.0f;
        total[j] = seg == 0 ? 0.0f : 1.0f;
    }
    if (!(MODE & kEnds)) {
        const float* e = r.ends + (static_cast<int64_t>(b) * r.plan.segments * in.D + my.c) * 2;
#pragma unroll 8
        for (int s = 0; s < seg; ++s, e += 2 * static_cast<int64_t>(in.D)) {
            const Pair made = *reinterpret_cast<const AnyPair*>(e);
#pragma unroll
            for (int j = 0; j < V; ++j) carry[j] = fmaf(made[2 * j], carry[j], made[2 * j + 1]);
        }
    }

    if (begin < end) {
        Bit<T, V> xr[P], fr[P], gr[P], zr[P];
        const auto fetch = [&](int l0) {
            take_rows<T, V, P>(fr, in.f, b, l0, len, bytes);
            take_rows<T, V, P>(gr, in.g, b, l0, len, bytes);
            take_rows<T, V, P>(xr, in.x, b, l0, len, bytes);
            if (GATED) take_rows<T, V, P>(zr, in.z, b, l0, len, bytes);
        };
        fetch(begin + w * P);
        int buffer = 0;
        for (int block = begin; block < end; block += W * P) {
            const int l0 = block + w * P;
            float a[P][V], put[P][V], h[V];
            Bit<T, V> z[P];
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const bool on = l0 + i < end;
                float x[V], f[V], g[V];
                xr[i].get(x);
                fr[i].get(f);
                gr[i].get(g);
                if (GATED) z[i] = zr[i];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const Decay d = decay_of(f[j], ch[j]);
                    a[i][j] = on ? d.a : 1.0f;
                    put[i][j] = on ? __builtin_amdgcn_sqrtf(d.rest) * sigmoid(g[j] + ch[j].g_bias) * x[j] : 0.0f;
                }
            }
            fetch(l0 + W * P);
            if constexpr (W > 1) {
                Pair mine;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float E = put[0][j];
#pragma unroll
                    for (int i = 1; i < P; ++i) E = fmaf(a[i][j], E, put[i][j]);
                    mine[2 * j] = product_of(a, j);
                    mine[2 * j + 1] = E;
                }
                pairs[buffer][w][lane] = mine;
                lds_sync();
#pragma unroll
                for (int k = 0; k < W; ++k) {
                    const Pair other = pairs[buffer][k][lane];
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        h[j] = k == w ? carry[j] : h[j];
                        carry[j] = fmaf(other[2 * j], carry[j], other[2 * j + 1]);
                        if (MODE & kEnds) total[j] = product(total[j], other[2 * j]);
                    }
                }
                buffer ^= 1;
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) h[j] = carry[j];
            }
            if ((MODE & kSave) && l0 % kRecurSave == 0 && l0 < end)
                my.give(r.saved + (static_cast<int64_t>(b) * ((in.N + kRecurSave - 1) / kRecurSave) + l0 / kRecurSave) * in.D, h);
            if constexpr ((MODE & kOut) != 0 || W == 1) {
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    float o[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) h[j] = fmaf(a[i][j], h[j], put[i][j]);
                    if (MODE & kOut) {
                        float zi[V];
                        if (GATED) z[i].get(zi);
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            o[j] = GATED ? h[j] * silu(zi[j]) : h[j];
                            o[j] = l0 + i < end ? o[j] : 0.0f;
                        }
                        if (l0 + i < stop) my.give(out + static_cast<int64_t>(l0 + i) * in.D, o);
                    }
                }
                if (W == 1) {
#pragma unroll
                    for (int j = 0; j < V; ++j) carry[j] = h[j];
                }
            }
        }
    }
    if (MODE & kOut) {
        const float zero[V] = {};
        const int done = begin < end ? begin + (end - begin + W * P - 1) / (W * P) * (W * P) : begin;
        for (int l = done + w; l < stop; l += W) my.give(out + static_cast<int64_t>(l) * in.D, zero);
    }
    if (w) return;
    if (MODE & kEnds) {
        float* e = r.ends + ((static_cast<int64_t>(b) * r.plan.segments + seg) * in.D + my.c) * 2;
        Pair made;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            made[2 * j] = total[j];
            made[2 * j + 1] = carry[j];
        }
        *reinterpret_cast<AnyPair*>(e) = made;  // (a channel that two lanes have: the same twice)
    } else if (r.final_state && end == len && (begin < len || seg == 0)) {
        my.give(r.final_state + static_cast<int64_t>(b) * in.D, carry);
    }
}

// ---- one position ---------------------------------------------------------------------------------------------
// A thread has W channels of one stream; their state is updated in place, so no two threads share one.
template <typename T, int W, bool GATED>
__global__ __launch_bounds__(256) void recur_step_kernel(RecurIn in, int cpr, float* __restrict__ state, T* __restrict__ out) {
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, b = id / cpr;
    if (b >= in.B) return;
    const int c = static_cast<int>(id - b * cpr) * W;
    Piece<T, W, W == 1> xr, fr, gr, zr;
    Piece<float, W, W == 1> sr;
    float* mine = state + b * in.D + c;
    xr.load(row_of<T>(in.x, b, 0) + c, W);
    fr.load(row_of<T>(in.f, b, 0) + c, W);
    gr.load(row_of<T>(in.g, b, 0) + c, W);
    if (GATED) zr.load(row_of<T>(in.z, b, 0) + c, W);
    sr.load(mine, W);
    float x[W], f[W], g[W], z[W], h[W], o[W];
    xr.get(x);
    fr.get(f);
    gr.get(g);
    if (GATED) zr.get(z);
    sr.get(h);
#pragma unroll
    for (int j = 0; j < W; ++j) {
        const RecurChannel ch = recur_channel(in, c + j);
        const Decay d = decay_of(f[j], ch);
        h[j] = fmaf(d.a, h[j], __builtin_amdgcn_sqrtf(d.rest) * sigmoid(g[j] + ch.g_bias) * x[j]);
        o[j] = GATED ? h[j] * silu(z[j]) : h[j];
    }
    Piece<float, W, W == 1>::put(mine, W, h);
    Piece<T, W, W == 1>::put(out + b * in.D + c, W, o);
}

template <typename T, int W>
hipError_t recur_step_of(const RecurIn& in, float* state, void* out, hipStream_t st) {
    const int cpr = in.D / W;
    const int64_t blocks = (static_cast<int64_t>(in.B) * cpr + 255) / 256;
    if (!fits(blocks, 256)) return hipErrorInvalidValue;
    const auto kernel = in.z.data ? recur_step_kernel<T, W, true> : recur_step_kernel<T, W, false>;
    kernel<<<static_cast<unsigned>(blocks), 256, 0, st>>>(in, cpr, state, static_cast<T*>(out));
    return hipGetLastError();
}

// ---- launches -------------------------------------------------------------------------------------------------

constexpr int kPositions = 8, kWaves = 8;  // a wave's and a workgroup's
static_assert(kRecurBlock % (kPositions * kWaves) == 0 && kRecurSave % kPositions == 0, "");

int channels_a_lane(int D) { return D == 1 ? 1 : 2; }

RecurPlan recur_plan(int B, int N, int D) {
    RecurPlan p;
    p.tiles = (D - 1) / (64 * channels_a_lane(D)) + 1;
    const int64_t groups = static_cast<int64_t>(B) * p.tiles, most = (static_cast<int64_t>(N) + 255) / 256;
    int64_t segments = groups <= 128 ? 512 / groups : 1;
    if (segments > most) segments = most;
    p.seg_len = static_cast<int>(((N + segments - 1) / segments + kRecurBlock - 1) / kRecurBlock * kRecurBlock);
    p.segments = static_cast<int>((static_cast<int64_t>(N) + p.seg_len - 1) / p.seg_len);
    return p;
}

template <typename T, int V, int W, int MODE>
hipError_t recur_launch(const RecurRun& r, hipStream_t st) {
    const bool gated = (MODE & kOut) && r.in.z.data;
    const auto kernel = gated ? recur_kernel<T, V, kPositions, W, MODE, (MODE & kOut) != 0> : recur_kernel<T, V, kPositions, W, MODE, false>;
    kernel<<<static_cast<unsigned>(static_cast<int64_t>(r.in.B) * r.plan.segments * r.plan.tiles), 64 * W, 0, st>>>(r);
    return hipGetLastError();
}
template <typename T, int V, int W>
hipError_t recur_of(const RecurRun& r, hipStream_t st) {
    if constexpr (W > 1) {
        if (r.plan.segments > 1)
            if (const hipError_t e = recur_launch<T, V, W, kEnds>(r, st); e != hipSuccess) return e;
    }
    if (!r.out) return recur_launch<T, V, W, kSave>(r, st);
    return r.saved ? recur_launch<T, V, W, kOut | kSave>(r, st) : recur_launch<T, V, W, kOut>(r, st);
}
template <typename T>
hipError_t recur_by(const RecurRun& r, hipStream_t st) {
    if (channels_a_lane(r.in.D) == 1) return r.in.N <= kPositions ? recur_of<T, 1, 1>(r, st) : recur_of<T, 1, kWaves>(r, st);
    return r.in.N <= kPositions ? recur_of<T, 2, 1>(r, st) : recur_of<T, 2, kWaves>(r, st);
}

}  // namespace

size_t recur_saved_bytes(int B, int N, int D) { return up256(static_cast<size_t>(B) * ((static_cast<int64_t>(N) + kRecurSave - 1) / kRecurSave) * D * 4); }

size_t recur_workspace(int B, int N, int D) {
    const RecurPlan p = recur_plan(B, N, D);
    return p.segments > 1 ? recur_ends_bytes(B, p.segments, D) : 256;
}

hipError_t launch_recur(int dtype, const RecurIn& in, const float* state, void* out, float* final_state, float* saved, void* ws, hipStream_t st) {
    const RecurRun r{in, state, out, final_state, saved, static_cast<float*>(ws), recur_plan(in.B, in.N, in.D)};
    if (!fits(static_cast<int64_t>(in.B) * r.plan.segments * r.plan.tiles, 64 * kWaves)) return hipErrorInvalidValue;
    return dtype ? recur_by<uint16_t>(r, st) : recur_by<float>(r, st);
}

hipError_t launch_recur_step(int dtype, const RecurIn& in, float* state, void* out, hipStream_t st) {
    if (in.D % 4 == 0) return dtype ? recur_step_of<uint16_t, 4>(in, state, out, st) : recur_step_of<float, 4>(in, state, out, st);
    return dtype ? recur_step_of<uint16_t, 1>(in, state, out, st) : recur_step_of<float, 1>(in, state, out, st);
}

}  // namespace enc
}  // namespace lccrf
