// Gradient of the gated linear recurrence.
//
// With dy = dout z s(z) and dh[l] = dy[l] + a[l+1] dh[l+1] running backwards, i = s(g), m = sqrt(1 - a^2), o = s(f):
//     dx = dh m i,   dg = dh m x i (1 - i),   dz = dout h (z s(z))',
//     dlog = dh (h[l-1] a u - i x a^2 u / m)   (by the logarithm of -u),   df = dlog (1 - o),   ddecay = sum dlog s(decay) / log(1 + exp(decay)).
// u / m goes to 0 with u, where 1 / m by itself does not.  As in the forward pass a workgroup's waves share a block of positions; they go
// backwards over the blocks, and (A, E) of every wave's positions is joined by G, what they turn a gradient c behind them into in front of
// them, A c + G.  The states in front of every block are saved by the forward pass, so one pass over the inputs is enough.
#include "lccrf_recur.h"

namespace lccrf {
namespace enc {
namespace {

constexpr int P = 4, W = 8;  // positions a wave, waves
static_assert(P * W == kRecurSave, "a block begins where a state is saved");

struct GradRun {
    RecurIn in;
    AnyRows dout;
    RecurGrads g;
    const float* saved;
    float* ends;     // segments > 1: [B][segments][D][2]: what a segment makes of a gradient behind it
    float* partial;  // [B * segments][3][D]: sums of dlog, df, dg
    RecurPlan plan;
};

template <typename T, int V, bool GATED, bool ENDS>
__global__ __launch_bounds__(64 * W) void recur_grad_kernel(GradRun r) {
    typedef float Four __attribute__((ext_vector_type(4)));
    typedef float Pair __attribute__((ext_vector_type(2 * V)));
    typedef Pair AnyPair __attribute__((aligned(4)));
    __shared__ Four made[2][W][V][64];  // A, E, G
    __shared__ float sums[ENDS ? 1 : W][3][V][64];
    const RecurIn& in = r.in;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned which = blockIdx.x / r.plan.tiles;
    const int tile = blockIdx.x - which * r.plan.tiles;
    const int b = which / r.plan.segments, seg = which - b * r.plan.segments;
    const Lane<V> my(tile, lane, in.D);
    const unsigned bytes = static_cast<unsigned>(my.c) * sizeof(T);
    const int len = length_at(in.lengths, b, in.N), begin = seg * r.plan.seg_len;
    const int stop = in.N - begin < r.plan.seg_len ? in.N : begin + r.plan.seg_len, end = stop < len ? stop : len;
    const int64_t first = static_cast<int64_t>(b) * in.N;

    RecurChannel ch[V];
    float behind[V], total[V], s_log[V], s_f[V], s_g[V];  // the gradient by the state behind the block; sums over this wave's positions
#pragma unroll
    for (int j = 0; j < V; ++j) {
        ch[j] = recur_channel(in, my.c + j);
        behind[j] = s_log[j] = s_f[j] = s_g[j] = 0.0f;
        total[j] = 1.0f;
    }
    if (!ENDS) {
        const int64_t base = static_cast<int64_t>(b) * r.plan.segments;
#pragma unroll 8
        for (int s = r.plan.segments - 1; s > seg; --s) {
            const Pair e = *reinterpret_cast<const AnyPair*>(r.ends + ((base + s) * in.D + my.c) * 2);
#pragma unroll
            for (int j = 0; j < V; ++j) behind[j] = fmaf(e[2 * j], behind[j], e[2 * j + 1]);
        }
        const float zero[V] = {};
        for (int l = (begin < end ? end : begin) + w; l < stop; l += W) {
            const int64_t at = (first + l) * in.D;
            my.give(static_cast<T*>(r.g.dx) + at, zero);
            my.give(static_cast<T*>(r.g.df) + at, zero);
            my.give(static_cast<T*>(r.g.dg) + at, zero);
            if (GATED) my.give(static_cast<T*>(r.g.dz) + at, zero);
        }
    }

    if (begin < end) {
        Bit<T, V> xr[P], fr[P], gr[P], zr[P], dr[P];
        Bit<float, V> sr;
        const auto fetch = [&](int block) {
            const int l0 = block + w * P;
            if (!ENDS) take_bit<float, V>(sr, r.saved + (static_cast<int64_t>(b) * ((in.N + kRecurSave - 1) / kRecurSave) + block / kRecurSave) * in.D, 4u * my.c);
            take_rows<T, V, P>(fr, in.f, b, l0, len, bytes);
            take_rows<T, V, P>(dr, r.dout, b, l0, len, bytes);
            if (GATED) take_rows<T, V, P>(zr, in.z, b, l0, len, bytes);
            if (!ENDS) {
                take_rows<T, V, P>(gr, in.g, b, l0, len, bytes);
                take_rows<T, V, P>(xr, in.x, b, l0, len, bytes);
            }
        };
        int block = begin + (end - begin - 1) / (P * W) * (P * W), buffer = 0;
        fetch(block);
        for (; block >= begin; block -= P * W) {
            const int l0 = block + w * P;
            float a[P][V], m[P][V], rest[P][V], open[P][V], in_gate[P][V], x[P][V], dy[P][V], h[V];
            Bit<T, V> z[P], dout[P];
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const bool on = l0 + i < end;
                float f[V], g[V], zi[V], di[V];
                fr[i].get(f);
                dr[i].get(di);
                dout[i] = dr[i];
                if (GATED) {
                    zr[i].get(zi);
                    z[i] = zr[i];
                }
                if (!ENDS) {
                    gr[i].get(g);
                    xr[i].get(x[i]);
                }
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const Decay d = decay_of(f[j], ch[j]);
                    a[i][j] = on ? d.a : 1.0f;
                    dy[i][j] = on ? GATED ? di[j] * silu(zi[j]) : di[j] : 0.0f;
                    if (!ENDS) {
                        open[i][j] = d.open;
                        rest[i][j] = d.rest;
                        m[i][j] = __builtin_amdgcn_sqrtf(d.rest);
                        in_gate[i][j] = sigmoid(g[j] + ch[j].g_bias);
                        x[i][j] = on ? x[i][j] : 0.0f;
                    }
                }
            }
            if (!ENDS) {
                float s[V];
                sr.get(s);
#pragma unroll
                for (int j = 0; j < V; ++j) h[j] = s[j];
            }
            fetch(block > begin ? block - P * W : begin);
            const auto put = [&](int i, int j) { return l0 + i < end ? m[i][j] * in_gate[i][j] * x[i][j] : 0.0f; };
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float G = 0.0f, E = 0.0f;
#pragma unroll
                for (int i = P - 1; i >= 0; --i) G = a[i][j] * (dy[i][j] + G);
                if (!ENDS) {
#pragma unroll
                    for (int i = 0; i < P; ++i) E = fmaf(a[i][j], E, put(i, j));
                }
                made[buffer][w][j][lane] = Four{product_of(a, j), E, G, 0.0f};
            }
            lds_sync();
            float c[V];  // the gradient behind this wave's positions
#pragma unroll
            for (int j = 0; j < V; ++j) {
                Four all[W];
#pragma unroll
                for (int k = 0; k < W; ++k) all[k] = made[buffer][k][j][lane];
#pragma unroll
                for (int k = W - 1; k >= 0; --k) {
                    c[j] = k == w ? behind[j] : c[j];
                    behind[j] = fmaf(all[k][0], behind[j], all[k][2]);
                    if (ENDS) total[j] = product(total[j], all[k][0]);
                }
                if (!ENDS) {
#pragma unroll
                    for (int k = 0; k < W - 1; ++k) h[j] = k < w ? fmaf(all[k][0], h[j], all[k][1]) : h[j];
                }
            }
            buffer ^= 1;
            if constexpr (!ENDS) {
                float before[P][V];
#pragma unroll
                for (int i = 0; i < P; ++i) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        before[i][j] = h[j];
                        h[j] = fmaf(a[i][j], h[j], put(i, j));
                    }
                }
#pragma unroll
                for (int i = P - 1; i >= 0; --i) {
                    float dx[V], df[V], dg[V], dz[V], zi[V], di[V];
                    dout[i].get(di);
                    if (GATED) z[i].get(zi);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float dh = dy[i][j] + c[j], u = ch[j].c * open[i][j], ai = a[i][j], gate_in = in_gate[i][j];
                        // u / m: 0 where 1 - a^2 is (or is too small for its root)
                        const float ratio = rest[i][j] < 1.17549435e-38f ? 0.0f : u * __builtin_amdgcn_rsqf(rest[i][j]);
                        dx[j] = dh * m[i][j] * gate_in;
                        dg[j] = dx[j] * x[i][j] * (1.0f - gate_in);
                        const float dlog = dh * ai * (before[i][j] * u - gate_in * x[i][j] * ai * ratio);
                        df[j] = dlog * (1.0f - open[i][j]);
                        if (GATED) {
                            const float gate = sigmoid(zi[j]);
                            dz[j] = di[j] * fmaf(ai, before[i][j], put(i, j)) * gate * fmaf(zi[j], 1.0f - gate, 1.0f);
                        }
                        c[j] = ai * dh;
                        const bool on = l0 + i < end;
                        s_log[j] += on ? dlog : 0.0f;
                        s_f[j] += on ? df[j] : 0.0f;
                        s_g[j] += on ? dg[j] : 0.0f;
                    }
                    if (l0 + i < end) {
                        const int64_t at = (first + l0 + i) * in.D;
                        my.give(static_cast<T*>(r.g.dx) + at, dx);
                        my.give(static_cast<T*>(r.g.df) + at, df);
                        my.give(static_cast<T*>(r.g.dg) + at, dg);
                        if (GATED) my.give(static_cast<T*>(r.g.dz) + at, dz);
                    }
                }
            }
        }
    }
    if constexpr (ENDS) {
        if (w) return;
        Pair e;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            e[2 * j] = total[j];
            e[2 * j + 1] = behind[j];
        }
        *reinterpret_cast<AnyPair*>(r.ends + ((static_cast<int64_t>(b) * r.plan.segments + seg) * in.D + my.c) * 2) = e;
    } else {
        if (w == 0 && seg == 0 && r.g.dstate) my.give(r.g.dstate + static_cast<int64_t>(b) * in.D, behind);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            sums[w][0][j][lane] = s_log[j];
            sums[w][1][j][lane] = s_f[j];
            sums[w][2][j][lane] = s_g[j];
        }
        lds_sync();
        if (w >= 3) return;
        float s[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            s[j] = sums[0][w][j][lane];
#pragma unroll
            for (int k = 1; k < W; ++k) s[j] += sums[k][w][j][lane];
        }
        my.give(r.partial + ((static_cast<int64_t>(b) * r.plan.segments + seg) * 3 + w) * in.D, s);
    }
}

// Sums over the sequences' segments: workgroups of 64 channels of one of the three, sixteen threads a channel.
__global__ __launch_bounds__(1024) void recur_sums_kernel(const float* __restrict__ partial, int64_t parts, int D, const float* __restrict__ decay, float* ddecay,
                                                          float* df_bias, float* dg_bias) {
    __shared__ float sums[16][64];
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6, k = blockIdx.y, ch = blockIdx.x * 64 + x;
    float* to = k == 0 ? ddecay : k == 1 ? df_bias : dg_bias;
    if (!to) return;
    float sum = 0.0f;
    if (ch < D)
        for (int64_t p = y; p < parts; p += 16) sum += partial[(p * 3 + k) * D + ch];
    sums[y][x] = sum;
    __syncthreads();
    if (y || ch >= D) return;
    for (int i = 1; i < 16; ++i) sum += sums[i][x];
    if (k == 0) {
        // s(decay) / log(1 + exp(decay)) is 1 - exp(decay) / 2 + ...: 1 in float from -17 down, where both go to 0 together
        const Softplus s = softplus(decay[ch]);
        sum *= decay[ch] < -17.0f ? 1.0f : s.slope / s.value;
    }
    to[ch] = sum;
}

int channels_a_lane(int D) { return D == 1 ? 1 : 2; }

RecurPlan grad_plan(int B, int N, int D) {
    RecurPlan p;
    p.tiles = (D - 1) / (64 * channels_a_lane(D)) + 1;
    const int64_t groups = static_cast<int64_t>(B) * p.tiles, most = (static_cast<int64_t>(N) + 255) / 256;
    int64_t segments = groups <= 128 ? 256 / groups : 1;
    if (segments > most) segments = most;
    p.seg_len = static_cast<int>(((N + segments - 1) / segments + kRecurBlock - 1) / kRecurBlock * kRecurBlock);
    p.segments = static_cast<int>((static_cast<int64_t>(N) + p.seg_len - 1) / p.seg_len);
    return p;
}

template <typename T, int V>
hipError_t grad_of(const GradRun& r, hipStream_t st) {
    const unsigned blocks = static_cast<unsigned>(static_cast<int64_t>(r.in.B) * r.plan.segments * r.plan.tiles);
    const bool gated = r.in.z.data != nullptr;
    if (r.plan.segments > 1) {
        const auto ends = gated ? recur_grad_kernel<T, V, true, true> : recur_grad_kernel<T, V, false, true>;
        ends<<<blocks, 64 * W, 0, st>>>(r);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    const auto kernel = gated ? recur_grad_kernel<T, V, true, false> : recur_grad_kernel<T, V, false, false>;
    kernel<<<blocks, 64 * W, 0, st>>>(r);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    recur_sums_kernel<<<dim3(pieces_of_row(r.in.D, 64), 3), 1024, 0, st>>>(r.partial, static_cast<int64_t>(r.in.B) * r.plan.segments, r.in.D, r.in.decay, r.g.ddecay,
                                                                             r.g.df_bias, r.g.dg_bias);
    return hipGetLastError();
}

size_t partial_bytes(int B, int segments, int D) { return up256(static_cast<size_t>(B) * segments * 3 * D * 4); }

}  // namespace

size_t recur_grad_workspace(int B, int N, int D, bool with_saved) {
    const RecurPlan p = grad_plan(B, N, D);
    size_t need = partial_bytes(B, p.segments, D) + (p.segments > 1 ? recur_ends_bytes(B, p.segments, D) : 0);
    if (!with_saved) need += recur_saved_bytes(B, N, D) + recur_workspace(B, N, D);
    return need;
}

hipError_t launch_recur_grad(int dtype, AnyRows dout, const RecurIn& in, const float* state, const float* saved, const RecurGrads& g, void* ws, hipStream_t st) {
    GradRun r{in, dout, g, saved, nullptr, static_cast<float*>(ws), grad_plan(in.B, in.N, in.D)};
    if (!fits(static_cast<int64_t>(in.B) * r.plan.segments * r.plan.tiles, 64 * W)) return hipErrorInvalidValue;
    char* more = static_cast<char*>(ws) + partial_bytes(in.B, r.plan.segments, in.D);
    if (r.plan.segments > 1) {
        r.ends = reinterpret_cast<float*>(more);
        more += recur_ends_bytes(in.B, r.plan.segments, in.D);
    }
    if (!saved) {
        r.saved = reinterpret_cast<float*>(more);
        if (const hipError_t e = launch_recur(dtype, in, state, nullptr, nullptr, reinterpret_cast<float*>(more), more + recur_saved_bytes(in.B, in.N, in.D), st); e != hipSuccess)
            return e;
    }
    if (in.D == 1) return dtype ? grad_of<uint16_t, 1>(r, st) : grad_of<float, 1>(r, st);
    return dtype ? grad_of<uint16_t, 2>(r, st) : grad_of<float, 2>(r, st);
}

}  // namespace enc
}  // namespace lccrf
