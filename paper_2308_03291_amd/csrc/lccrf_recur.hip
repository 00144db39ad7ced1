// Gated linear recurrence: forward pass and single-token form (lccrf_recur.h says how the work is spread).
#include "lccrf_recur.h"

#include <type_traits>

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
    float* ends;   // segments > 1: [B][segments][D][2]: what a segment makes of a state (kEnds: written); the first one: the call's state, and what it makes of it
    RecurPlan plan;
};

template <typename T, int V, int P, int W, int SUB, int MODE, bool GATED>
__global__ __launch_bounds__(64 * W) void recur_kernel(RecurRun r) {
    constexpr int L = 64 / SUB, kRows = SUB * P, kBlock = W * kRows;  // lanes across the tile; positions a wave and a block
    typedef float Pair __attribute__((ext_vector_type(2 * V)));
    typedef Pair AnyPair __attribute__((aligned(4)));
    typedef float Some __attribute__((ext_vector_type(V)));
    __shared__ Pair pairs[W > 1 ? 2 : 1][W][L];
    __shared__ Some states[W > 1 ? 2 : 1][L];  // in front of the block
    const RecurIn& in = r.in;
    const int lane = threadIdx.x & 63, cl = lane % L, w = W > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const int sub = lane / L, set = sub * P;
    const RecurWork work = recur_work(r.plan);
    const int b = work.b, seg = work.seg;
    if (b >= in.B) return;
    const Lane<V> my(work.tile, cl, L, in.D);
    const int len = length_at(in.lengths, b, in.N), begin = seg * r.plan.seg_len;
    const int stop = in.N - begin < r.plan.seg_len ? in.N : begin + r.plan.seg_len, end = stop < len ? stop : len;
    T* out = static_cast<T*>(r.out) + static_cast<int64_t>(b) * in.N * in.D;

    // (where sequences are cut the second pass takes the call's state from `ends`: a later segment may have written the final one over it already)
    const bool cut = !(MODE & kEnds) && r.plan.segments > 1;
    RecurChannel ch[V];
    float carry[V], total[V];  // the state in front of the first block, later (the last lanes': behind their positions) of the next one; kEnds: this lane's product of decays
#pragma unroll
    for (int j = 0; j < V; ++j) {
        ch[j] = recur_channel(in, my.c + j);
        carry[j] = seg == 0 && r.state && !cut ? r.state[static_cast<int64_t>(b) * in.D + my.c + j] : 0.0f;
        total[j] = 1.0f;
    }
    if (cut && seg == 0 && r.state) {
        const Pair made = *reinterpret_cast<const AnyPair*>(r.ends + (static_cast<int64_t>(b) * r.plan.segments * in.D + my.c) * 2);
#pragma unroll
        for (int j = 0; j < V; ++j) carry[j] = made[2 * j];
    }
    const bool last = w == W - 1 && sub == SUB - 1;

    if (begin < end) {
        Bit<T, V> xr[P], fr[P], gr[P], zr[P];
        const auto fetch = [&](int first, auto whole) {
            constexpr bool WHOLE = decltype(whole)::value;
            unsigned bytes = static_cast<unsigned>(my.c) * sizeof(T);
            asm volatile("" : "+v"(bytes));  // added by the loads themselves, not to every input's address ahead of the loop
            take_rows<T, V, P, SUB, WHOLE>(fr, in.f, b, first, len, set, bytes);
            take_rows<T, V, P, SUB, WHOLE>(gr, in.g, b, first, len, set, bytes);
            take_rows<T, V, P, SUB, WHOLE>(xr, in.x, b, first, len, set, bytes);
            if (GATED) take_rows<T, V, P, SUB, WHOLE>(zr, in.z, b, first, len, set, bytes);
        };
        fetch(begin + w * kRows, std::false_type{});
        if constexpr (!(MODE & kEnds) && W > 1) {
            // the segments in front, a share of them a wave, on top of the first loads
            if (seg > 0) {
                const int share = (seg + W - 1) / W, from = w * share, to = seg < from + share ? seg : from + share;
                const float* e = r.ends + ((static_cast<int64_t>(b) * r.plan.segments + from) * in.D + my.c) * 2;
                Pair mine;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    mine[2 * j] = 1.0f;
                    mine[2 * j + 1] = 0.0f;
                }
#pragma unroll 8
                for (int s = from; s < to; ++s, e += 2 * static_cast<int64_t>(in.D)) {
                    const Pair made = *reinterpret_cast<const AnyPair*>(e);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float a = s > 0 ? made[2 * j] : 0.0f;
                        mine[2 * j] = product(mine[2 * j], a);
                        mine[2 * j + 1] = fmaf(a, mine[2 * j + 1], made[2 * j + 1]);
                    }
                }
                if (sub == 0) pairs[1][w][cl] = mine;  // (the other buffer than the first block's)
                lds_sync();
#pragma unroll
                for (int k = 0; k < W; ++k) {
                    const Pair made = pairs[1][k][cl];
#pragma unroll
                    for (int j = 0; j < V; ++j) carry[j] = fmaf(made[2 * j], carry[j], made[2 * j + 1]);
                }
            }
        }
        int buffer = 0;
        const auto leave = [&](int to) {
            Some s;
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] = carry[j];
            if (last) states[to][cl] = s;
        };
        if (W > 1) leave(0);
        // whole: all positions lie before the end; ahead: and so do the next block's; full: all lanes have V channels of their own
        const auto run = [&](auto whole, auto ahead, auto full, int first) {
            constexpr bool WHOLE = decltype(whole)::value, FULL = decltype(full)::value;
            const int l0 = first + set;
            float a[P][V], put[P][V];
            float(&h)[V] = carry;
            Bit<T, V> z[P];
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const bool on = WHOLE || l0 + i < end;
                float x[V], f[V], g[V];
                xr[i].get(x);
                fr[i].get(f);
                gr[i].get(g);
                if (GATED) z[i] = zr[i];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const Decay d = decay_of(f[j], ch[j]);
                    a[i][j] = on ? d.a : 1.0f;
                    put[i][j] = on ? __builtin_amdgcn_sqrtf(d.rest) * open_gate(g[j], ch[j].g_bias) * x[j] : 0.0f;
                }
            }
            if (decltype(ahead)::value || first + kBlock < end) fetch(first + kBlock, ahead);
            if constexpr (W > 1) {
                Pair mine;
                float A[V], E[V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    E[j] = put[0][j];
#pragma unroll
                    for (int i = 1; i < P; ++i) E[j] = fmaf(a[i][j], E[j], put[i][j]);
                    A[j] = product_of(a, j);
                    if (MODE & kEnds) total[j] = product(total[j], A[j]);
                    const float own_a = A[j], own_e = E[j];
                    before_set<SUB, false>(A[j], E[j], sub);
                    mine[2 * j] = SUB > 1 ? product(own_a, A[j]) : own_a;
                    mine[2 * j + 1] = SUB > 1 ? fmaf(own_a, E[j], own_e) : own_e;
                }
                if (SUB == 1 || sub == SUB - 1) pairs[buffer][w][cl] = mine;
                lds_sync();
                Pair others[W - 1];
                const Some from = states[buffer][cl];
#pragma unroll
                for (int k = 0; k < W - 1; ++k) others[k] = pairs[buffer][k][cl];
#pragma unroll
                for (int j = 0; j < V; ++j) h[j] = from[j];
#pragma unroll
                for (int k = 0; k < W - 1; ++k) {
                    if (k == w) break;
#pragma unroll
                    for (int j = 0; j < V; ++j) h[j] = fmaf(others[k][2 * j], h[j], others[k][2 * j + 1]);
                }
                if (SUB > 1) {
#pragma unroll
                    for (int j = 0; j < V; ++j) h[j] = fmaf(A[j], h[j], E[j]);
                }
                buffer ^= 1;
            }
            if ((MODE & kSave) && l0 % kRecurSave == 0 && l0 < end)
                my.template give<FULL>(r.saved + (static_cast<int64_t>(b) * ((in.N + kRecurSave - 1) / kRecurSave) + l0 / kRecurSave) * in.D, h);
            if constexpr ((MODE & kOut) != 0 || W == 1) {
                // a place for the whole wave and the lane's offset in it
                T* to = out + static_cast<int64_t>(first) * in.D;
                const unsigned at = static_cast<unsigned>(set) * static_cast<unsigned>(in.D);
#pragma unroll
                for (int i = 0; i < P; ++i, to += in.D) {
                    float o[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) h[j] = fmaf(a[i][j], h[j], put[i][j]);
                    if (MODE & kOut) {
                        float zi[V];
                        if (GATED) z[i].get(zi);
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            o[j] = GATED ? h[j] * silu(zi[j]) : h[j];
                            o[j] = WHOLE || l0 + i < end ? o[j] : 0.0f;
                        }
                        if (WHOLE || l0 + i < stop) my.template give<FULL>(to, o, SUB > 1 ? at : 0u);
                    }
                }
            } else if (w == W - 1) {
#pragma unroll
                for (int i = 0; i < P; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j) h[j] = fmaf(a[i][j], h[j], put[i][j]);
            }
            if (W > 1) leave(buffer);
        };
        int block = begin;
        const auto whole_blocks = [&](auto full) {
            for (; block + 2 * kBlock <= end; block += kBlock) run(std::true_type{}, std::true_type{}, full, block + w * kRows);
            if (block + kBlock <= end) {
                run(std::true_type{}, std::false_type{}, full, block + w * kRows);
                block += kBlock;
            }
        };
        if (my.full || (MODE & kEnds)) whole_blocks(std::true_type{});  // (which gives nothing away here)
        else whole_blocks(std::false_type{});
        for (; block < end; block += kBlock) run(std::false_type{}, std::false_type{}, std::false_type{}, block + w * kRows);
    }
    if (MODE & kOut) {
        const float zero[V] = {};
        const int done = begin < end ? begin + (end - begin + kBlock - 1) / kBlock * kBlock : begin;
        for (int l = done + w * SUB + sub; l < stop; l += W * SUB) my.give(out + static_cast<int64_t>(l) * in.D, zero);
    }
    if constexpr ((MODE & kEnds) != 0) {
        // the product over all lanes of a channel, each with its positions of all blocks
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int d = L; d < 64; d *= 2) total[j] = product(total[j], __shfl_xor(total[j], d));
        lds_sync();
        if (sub == 0) {
#pragma unroll
            for (int j = 0; j < V; ++j) pairs[0][w][cl][j] = total[j];
        }
        lds_sync();
        if (!last) return;
        Pair made;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float all = 1.0f;
#pragma unroll
            for (int k = 0; k < W; ++k) all = product(all, pairs[0][k][cl][j]);
            made[2 * j] = seg > 0 ? all : r.state ? r.state[static_cast<int64_t>(b) * in.D + my.c + j] : 0.0f;
            made[2 * j + 1] = carry[j];
        }
        *reinterpret_cast<AnyPair*>(r.ends + ((static_cast<int64_t>(b) * r.plan.segments + seg) * in.D + my.c) * 2) = made;  // (a channel of two lanes: the same twice)
    } else if (last && r.final_state && end == len && (begin < len || seg == 0)) {
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
        h[j] = fmaf(d.a, h[j], __builtin_amdgcn_sqrtf(d.rest) * open_gate(g[j], ch.g_bias) * x[j]);
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

constexpr int kPositions = 4, kWaves = 8, kFewWaves = 4;  // a lane's positions; a workgroup's waves, and where sequences are cut

int channels_a_lane(int D) { return D == 1 ? 1 : 2; }

// Measured, us, wide tiles / narrow / segments (B x N x D, bfloat16, no gate but in the first): 64x512x2048 145 / 158 / 252, 16x1000x1024 51 / 47 / 54, 30x300x300
// 21 / 18 / 21, 8x256x1024 16 / 14 / 19, 4x5000x1024 228 / 91 / 64, 2x10000x256 446 / 143 / 29, 4x16384x514 865 / 263 / 118.  The first is 4.65 TB/s (float 5.5;
// a copy, which writes as much as it reads, 5.14); segments are read twice: the last one's two passes take 56 us (3.6 TB/s) and 60 (4.5).
static_assert(kWaves != kFewWaves, "workgroups of so few have segments");
RecurPlan recur_plan(int B, int N, int D) { return recur_plan_of(B, N, D, 256, 256, 512); }

template <typename T, int V, int W, int SUB, int MODE>
hipError_t recur_launch(const RecurRun& r, hipStream_t st) {
    const bool gated = (MODE & kOut) && r.in.z.data;
    const auto kernel = gated ? recur_kernel<T, V, kPositions, W, SUB, MODE, (MODE & kOut) != 0> : recur_kernel<T, V, kPositions, W, SUB, MODE, false>;
    kernel<<<static_cast<unsigned>(recur_blocks(r.plan, r.in.B)), 64 * W, 0, st>>>(r);
    return hipGetLastError();
}
template <typename T, int V, int W, int SUB>
hipError_t recur_of(const RecurRun& r, hipStream_t st) {
    if constexpr (W == kFewWaves)
        if (const hipError_t e = recur_launch<T, V, W, SUB, kEnds>(r, st); e != hipSuccess) return e;
    if (!r.out) return recur_launch<T, V, W, SUB, kSave>(r, st);
    return r.saved ? recur_launch<T, V, W, SUB, kOut | kSave>(r, st) : recur_launch<T, V, W, SUB, kOut>(r, st);
}
template <typename T, int V>
hipError_t recur_by(const RecurRun& r, hipStream_t st) {
    if (r.plan.segments > 1) return recur_of<T, V, kFewWaves, 1>(r, st);
    if (r.in.N <= kPositions) return recur_of<T, V, 1, 1>(r, st);
    if constexpr (V > 1) {
        if (r.plan.narrow) return recur_of<T, V, kWaves, 4>(r, st);
    }
    return recur_of<T, V, kWaves, 1>(r, st);
}

}  // namespace

size_t recur_saved_bytes(int B, int N, int D) { return up256(static_cast<size_t>(B) * ((static_cast<int64_t>(N) + kRecurSave - 1) / kRecurSave) * D * 4); }

size_t recur_workspace(int B, int N, int D) {
    const RecurPlan p = recur_plan(B, N, D);
    return p.segments > 1 ? recur_ends_bytes(B, p.segments, D) : 0;
}

hipError_t launch_recur(int dtype, const RecurIn& in, const float* state, void* out, float* final_state, float* saved, void* ws, hipStream_t st) {
    RecurRun r{in, state, out, final_state, saved, static_cast<float*>(ws), recur_plan(in.B, in.N, in.D)};
    if (in.N <= kPositions || !near_rows(in.x) || !near_rows(in.f) || !near_rows(in.g) || !near_rows(in.z)) widen_tiles(r.plan, in.D);
    if (!fits(recur_blocks(r.plan, in.B), 64 * kWaves)) return hipErrorInvalidValue;
    if (channels_a_lane(in.D) == 1) return dtype ? recur_by<uint16_t, 1>(r, st) : recur_by<float, 1>(r, st);
    return dtype ? recur_by<uint16_t, 2>(r, st) : recur_by<float, 2>(r, st);
}

hipError_t launch_recur_step(int dtype, const RecurIn& in, float* state, void* out, hipStream_t st) {
    if (in.D % 4 == 0) return dtype ? recur_step_of<uint16_t, 4>(in, state, out, st) : recur_step_of<float, 4>(in, state, out, st);
    return dtype ? recur_step_of<uint16_t, 1>(in, state, out, st) : recur_step_of<float, 1>(in, state, out, st);
}

}  // namespace enc
}  // namespace lccrf
