// Gradient of the gated linear recurrence.
//
// With dy = dout z s(z) and dh[l] = dy[l] + a[l+1] dh[l+1] running backwards, i = s(g), m = sqrt(1 - a^2), o = s(f):
//     dx = dh m i,   dg = dh m x i (1 - i),   dz = dout h (z s(z))',
//     dlog = dh (h[l-1] a u - i x a^2 u / m)   (by the logarithm of -u),   df = dlog (1 - o),   ddecay = sum dlog s(decay) / log(1 + exp(decay)).
// u / m goes to 0 with u, where 1 / m by itself does not.  As in the forward pass a workgroup's waves share a block of positions; they go
// backwards over the blocks, and (A, E) of every wave's positions is joined by G, what they turn a gradient c behind them into in front of
// them, A c + G.  The states in front of every block are saved by the forward pass, so one pass over the inputs is enough.
#include "lccrf_recur.h"

#include <type_traits>

namespace lccrf {
namespace enc {
namespace {

struct GradRun {
    RecurIn in;
    AnyRows dout;
    RecurGrads g;
    const float* saved;
    float* ends;     // segments > 1: [B][segments][D][2]: what a segment makes of a gradient behind it
    float* partial;  // [B * segments][3][D]: sums of dlog, df, dg
    RecurPlan plan;
};

template <typename T, int V, int P, int W, int SUB, bool GATED, bool ENDS>
__global__ __launch_bounds__(64 * W) void recur_grad_kernel(GradRun r) {
    constexpr int L = 64 / SUB, kRows = SUB * P, kBlock = W * kRows;
    typedef float Three __attribute__((ext_vector_type(4)));
    typedef float Pair __attribute__((ext_vector_type(2 * V)));
    typedef Pair AnyPair __attribute__((aligned(4)));
    __shared__ Three made[2][W][V][L];  // A, E, G
    __shared__ float behinds[2][V][L];
    __shared__ float sums[ENDS ? 1 : W][3][V][L];
    const RecurIn& in = r.in;
    const int lane = threadIdx.x & 63, cl = lane % L, sub = lane / L, set = sub * P, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const RecurWork work = recur_work(r.plan);
    const int b = work.b, seg = work.seg;
    if (b >= in.B) return;
    const Lane<V> my(work.tile, cl, L, in.D);
    const int len = length_at(in.lengths, b, in.N), begin = seg * r.plan.seg_len;
    const int stop = in.N - begin < r.plan.seg_len ? in.N : begin + r.plan.seg_len, end = stop < len ? stop : len;
    const int64_t first_row = static_cast<int64_t>(b) * in.N;
    const bool front = w == 0 && sub == 0;

    RecurChannel ch[V];
    float c[V], total[V], s_log[V], s_f[V], s_g[V];  // the gradient behind (the front lanes': the next) block; this lane's product and sums
#pragma unroll
    for (int j = 0; j < V; ++j) {
        ch[j] = recur_channel(in, my.c + j);
        c[j] = s_log[j] = s_f[j] = s_g[j] = 0.0f;
        total[j] = 1.0f;
    }
    if (!ENDS) {
        const float zero[V] = {};
        for (int l = (begin < end ? end : begin) + w * SUB + sub; l < stop; l += W * SUB) {
            const int64_t at = (first_row + l) * in.D;
            my.give(static_cast<T*>(r.g.dx) + at, zero);
            my.give(static_cast<T*>(r.g.df) + at, zero);
            my.give(static_cast<T*>(r.g.dg) + at, zero);
            if (GATED) my.give(static_cast<T*>(r.g.dz) + at, zero);
        }
    }

    if (begin < end) {
        Bit<T, V> xr[P], fr[P], gr[P], zr[P], dr[P];
        Bit<float, V> sr;
        const auto fetch = [&](int block, auto whole) {
            constexpr bool WHOLE = decltype(whole)::value;
            const int first = block + w * kRows;
            unsigned bytes = static_cast<unsigned>(my.c) * sizeof(T);
            asm volatile("" : "+v"(bytes));  // added by the load itself, not to every row's address ahead of the loop
            if (!ENDS) take_bit<float, V>(sr, r.saved + (static_cast<int64_t>(b) * ((in.N + kRecurSave - 1) / kRecurSave) + block / kRecurSave) * in.D, 4u * my.c);
            take_rows<T, V, P, SUB, WHOLE>(fr, in.f, b, first, len, set, bytes);
            take_rows<T, V, P, SUB, WHOLE>(dr, r.dout, b, first, len, set, bytes);
            if (GATED) take_rows<T, V, P, SUB, WHOLE>(zr, in.z, b, first, len, set, bytes);
            if (!ENDS) {
                take_rows<T, V, P, SUB, WHOLE>(gr, in.g, b, first, len, set, bytes);
                take_rows<T, V, P, SUB, WHOLE>(xr, in.x, b, first, len, set, bytes);
            }
        };
        int block = begin + (end - begin - 1) / kBlock * kBlock;
        fetch(block, std::false_type{});
        if (!ENDS && len > stop) {
            // the segments behind that have positions, a share of them a wave, on top of the first loads
            const int many = (len - stop - 1) / r.plan.seg_len + 1, share = (many + W - 1) / W, from = w * share, to = many < from + share ? many : from + share;
            const float* e = r.ends + ((static_cast<int64_t>(b) * r.plan.segments + seg + to) * in.D + my.c) * 2;
            float A[V], G[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                A[j] = 1.0f;
                G[j] = 0.0f;
            }
#pragma unroll 8
            for (int s = to; s > from; --s, e -= 2 * static_cast<int64_t>(in.D)) {
                const Pair made_there = *reinterpret_cast<const AnyPair*>(e);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    A[j] = product(A[j], made_there[2 * j]);
                    G[j] = fmaf(made_there[2 * j], G[j], made_there[2 * j + 1]);
                }
            }
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (sub == 0) made[1][w][j][cl] = Three{A[j], 0.0f, G[j], 0.0f};  // (the other buffer than the first block's)
            lds_sync();
#pragma unroll
            for (int k = W - 1; k >= 0; --k)
#pragma unroll
                for (int j = 0; j < V; ++j) c[j] = fmaf(made[1][k][j][cl][0], c[j], made[1][k][j][cl][2]);
        }
        int buffer = 0;
        const auto leave = [&](int to) {
            if (front) {
#pragma unroll
                for (int j = 0; j < V; ++j) behinds[to][j][cl] = c[j];
            }
        };
        leave(0);
        const auto run = [&](auto whole, auto full, int block) {  // whole: all positions lie before the end; full: all lanes have V channels of their own
            constexpr bool WHOLE = decltype(whole)::value, FULL = decltype(full)::value;
            const int first = block + w * kRows, l0 = first + set;
            float a[P][V], m[P][V], inv[P][V], open[P][V], in_gate[P][V], x[P][V], dy[P][V], h[V];
            Bit<T, V> z[P], dout[P];
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const bool on = WHOLE || l0 + i < end;
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
                        // u / m is 0 where 1 - a^2 is (or is too small for its root)
                        inv[i][j] = d.rest < 1.17549435e-38f ? 0.0f : __builtin_amdgcn_rsqf(d.rest);
                        m[i][j] = d.rest * inv[i][j];
                        in_gate[i][j] = open_gate(g[j], ch[j].g_bias);
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
            fetch(block > begin ? block - kBlock : begin, whole);  // (whole: so are those in front)
            const auto put = [&](int i, int j) { return WHOLE || l0 + i < end ? m[i][j] * in_gate[i][j] * x[i][j] : 0.0f; };
            float before_a[V], before_e[V], behind_a[V], behind_g[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float G = 0.0f, E = 0.0f;
#pragma unroll
                for (int i = P - 1; i >= 0; --i) G = a[i][j] * (dy[i][j] + G);
                const float A = product_of(a, j);
                if (ENDS) total[j] = product(total[j], A);
                behind_a[j] = A;
                behind_g[j] = G;
                before_set<SUB, true>(behind_a[j], behind_g[j], sub);
                if (!ENDS) {
#pragma unroll
                    for (int i = 0; i < P; ++i) E = fmaf(a[i][j], E, put(i, j));
                    before_a[j] = A;
                    before_e[j] = E;
                    before_set<SUB, false>(before_a[j], before_e[j], sub);
                }
                // a wave's: the last set's way forwards, the first one's backwards
                if (SUB == 1) {
                    made[buffer][w][j][cl] = Three{A, E, G, 0.0f};
                } else {
                    if (sub == 0) {
                        made[buffer][w][j][cl][0] = product(A, behind_a[j]);
                        made[buffer][w][j][cl][2] = fmaf(A, behind_g[j], G);
                    }
                    if (!ENDS && sub == SUB - 1) made[buffer][w][j][cl][1] = fmaf(A, before_e[j], E);
                }
            }
            lds_sync();
#pragma unroll
            for (int j = 0; j < V; ++j) {
                Three all[W];
                c[j] = behinds[buffer][j][cl];
#pragma unroll
                for (int k = 0; k < W; ++k) all[k] = made[buffer][k][j][cl];
#pragma unroll
                for (int k = W - 1; k > 0; --k) {
                    if (k == w) break;
                    c[j] = fmaf(all[k][0], c[j], all[k][2]);
                }
                if (SUB > 1) c[j] = fmaf(behind_a[j], c[j], behind_g[j]);
                if (!ENDS) {
#pragma unroll
                    for (int k = 0; k < W - 1; ++k) {
                        if (k == w) break;
                        h[j] = fmaf(all[k][0], h[j], all[k][1]);
                    }
                    if (SUB > 1) h[j] = fmaf(before_a[j], h[j], before_e[j]);
                }
            }
            buffer ^= 1;
            if constexpr (ENDS) {
                if (w == 0) {
#pragma unroll
                    for (int i = P - 1; i >= 0; --i)
#pragma unroll
                        for (int j = 0; j < V; ++j) c[j] = a[i][j] * (dy[i][j] + c[j]);
                }
            } else {
                float before[P][V];
#pragma unroll
                for (int i = 0; i < P; ++i) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        before[i][j] = h[j];
                        h[j] = fmaf(a[i][j], h[j], put(i, j));
                    }
                }
                const unsigned at = SUB > 1 ? static_cast<unsigned>(set) * static_cast<unsigned>(in.D) : 0u;
#pragma unroll
                for (int i = P - 1; i >= 0; --i) {
                    float dx[V], df[V], dg[V], dz[V], zi[V], di[V];
                    const bool on = WHOLE || l0 + i < end;
                    dout[i].get(di);
                    if (GATED) z[i].get(zi);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float dh = dy[i][j] + c[j], u = kLn2f * (ch[j].c * open[i][j]), ai = a[i][j], gate_in = in_gate[i][j];
                        dx[j] = dh * m[i][j] * gate_in;
                        dg[j] = dx[j] * x[i][j] * (1.0f - gate_in);
                        const float dlog = dh * ai * (before[i][j] * u - gate_in * x[i][j] * ai * (u * inv[i][j]));
                        df[j] = dlog * (1.0f - open[i][j]);
                        if (GATED) {
                            const float gate = sigmoid(zi[j]);
                            dz[j] = di[j] * fmaf(ai, before[i][j], put(i, j)) * gate * fmaf(zi[j], 1.0f - gate, 1.0f);
                        }
                        c[j] = ai * dh;
                        s_log[j] += on ? dlog : 0.0f;
                        s_f[j] += on ? df[j] : 0.0f;
                        s_g[j] += on ? dg[j] : 0.0f;
                    }
                    if (on) {
                        const int64_t row = (first_row + first + i) * in.D;
                        my.template give<FULL>(static_cast<T*>(r.g.dx) + row, dx, at);
                        my.template give<FULL>(static_cast<T*>(r.g.df) + row, df, at);
                        my.template give<FULL>(static_cast<T*>(r.g.dg) + row, dg, at);
                        if (GATED) my.template give<FULL>(static_cast<T*>(r.g.dz) + row, dz, at);
                    }
                }
            }
            leave(buffer);
        };
        if (block + kBlock > end) {
            run(std::false_type{}, std::false_type{}, block);
            block -= kBlock;
        }
        if (my.full || ENDS) {  // (which give nothing away)
            for (; block >= begin; block -= kBlock) run(std::true_type{}, std::true_type{}, block);
        } else {
            for (; block >= begin; block -= kBlock) run(std::true_type{}, std::false_type{}, block);
        }
    }
    if constexpr (ENDS) {
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int d = L; d < 64; d *= 2) total[j] = product(total[j], __shfl_xor(total[j], d));
        lds_sync();
        if (sub == 0) {
#pragma unroll
            for (int j = 0; j < V; ++j) made[0][w][j][cl][0] = total[j];
        }
        lds_sync();
        if (!front) return;
        Pair e;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float all = 1.0f;
#pragma unroll
            for (int k = 0; k < W; ++k) all = product(all, made[0][k][j][cl][0]);
            e[2 * j] = all;
            e[2 * j + 1] = c[j];
        }
        *reinterpret_cast<AnyPair*>(r.ends + ((static_cast<int64_t>(b) * r.plan.segments + seg) * in.D + my.c) * 2) = e;
    } else {
        if (front && seg == 0 && r.g.dstate) my.give(r.g.dstate + static_cast<int64_t>(b) * in.D, c);
#pragma unroll
        for (int j = 0; j < V; ++j) {
#pragma unroll
            for (int d = L; d < 64; d *= 2) {
                s_log[j] += __shfl_xor(s_log[j], d);
                s_f[j] += __shfl_xor(s_f[j], d);
                s_g[j] += __shfl_xor(s_g[j], d);
            }
            if (sub == 0) {
                sums[w][0][j][cl] = s_log[j];
                sums[w][1][j][cl] = s_f[j];
                sums[w][2][j][cl] = s_g[j];
            }
        }
        lds_sync();
        if (w >= 3 || sub) return;
        float s[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            s[j] = sums[0][w][j][cl];
#pragma unroll
            for (int k = 1; k < W; ++k) s[j] += sums[k][w][j][cl];
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

constexpr int P = 2, W = 4;  // a lane's positions, a workgroup's waves: 125 registers (bfloat16), four waves a SIMD, so that the 1024 workgroups of B=128 N=256
                             // D=1024 run at once (whole training step, ragged, us: 188 - 194; at 142 registers 203 - 210; four positions, 203 registers, 227)
static_assert(P * W % kRecurSave == 0, "a block begins where a state is saved");

// Measured, us, forward and gradient, wide tiles / narrow / segments (B x N x D, bfloat16): 128x256x1024 ragged 188 / 219 / 267, 64x1024x514 371 / 354 / 384 (forwards
// wide, backwards segments: 355), 16x1000x1024 222 / 164 / 156 (forwards narrow: 151), 100x200x128 59 / 48 / 61, 30x300x300 89 / 61 / 61, 8x256x1024 69 / 51 / 61,
// 4x5000x1024 1057 / 447 / 193.
RecurPlan grad_plan(int B, int N, int D) { return recur_plan_of(B, N, D, 768, 1 << 30, 512); }

template <typename T, int V, int SUB>
hipError_t grad_of(const GradRun& r, hipStream_t st) {
    const unsigned blocks = static_cast<unsigned>(recur_blocks(r.plan, r.in.B));
    const bool gated = r.in.z.data != nullptr;
    if constexpr (SUB == 1) {
        if (r.plan.segments > 1) {
            const auto ends = gated ? recur_grad_kernel<T, V, P, W, SUB, true, true> : recur_grad_kernel<T, V, P, W, SUB, false, true>;
            ends<<<blocks, 64 * W, 0, st>>>(r);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        }
    }
    const auto kernel = gated ? recur_grad_kernel<T, V, P, W, SUB, true, false> : recur_grad_kernel<T, V, P, W, SUB, false, false>;
    kernel<<<blocks, 64 * W, 0, st>>>(r);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    recur_sums_kernel<<<dim3(pieces_of_row(r.in.D, 64), 3), 1024, 0, st>>>(r.partial, static_cast<int64_t>(r.in.B) * r.plan.segments, r.in.D, r.in.decay, r.g.ddecay,
                                                                             r.g.df_bias, r.g.dg_bias);
    return hipGetLastError();
}
template <typename T, int V>
hipError_t grad_by(const GradRun& r, hipStream_t st) {
    if constexpr (V > 1) {
        if (r.plan.narrow) return grad_of<T, V, 4>(r, st);
    }
    return grad_of<T, V, 1>(r, st);
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
    if (!near_rows(in.x) || !near_rows(in.f) || !near_rows(in.g) || !near_rows(in.z) || !near_rows(dout)) widen_tiles(r.plan, in.D);
    if (!fits(recur_blocks(r.plan, in.B), 64 * W)) return hipErrorInvalidValue;
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
    if (in.D == 1) return dtype ? grad_by<uint16_t, 1>(r, st) : grad_by<float, 1>(r, st);
    return dtype ? grad_by<uint16_t, 2>(r, st) : grad_by<float, 2>(r, st);
}

}  // namespace enc
}  // namespace lccrf
