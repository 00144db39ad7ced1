// Selective state space scan: forward pass and single-token form.
//
// An update of one state is a product, an exponential (two issue slots), a product, two fused multiply-adds: six slots of a
// SIMD, which with 16 states bound the pass before its traffic does (a channel and position takes 96 slots and some 30 for step and
// gate, against 8 bytes).  All of it is vector arithmetic: the decays differ by channel and state, so no matrix instruction has the form.
// Measured (B=64 N=512 D=2048 S=16, bfloat16, gated): 256 us, 2.1 TB/s; 116 vector instructions a channel and position, the vector
// pipes busy 92 % of the time, at the 2.0 GHz that the card keeps under this load.
// Segments of a sequence run side by side where the batch is small (scan_plan).
#include "lccrf_state.h"

namespace lccrf {
namespace enc {
namespace {

enum { kOut = 1, kSave = 2, kEnds = 4 };

struct ScanRun {
    ScanIn in;
    const float* state;  // [B][D][S] or null
    void* out;
    float* final_state;
    float* saved;
    float* ends;   // segments > 1: the states in front of every segment (kEnds: written, what a segment makes of 0)
    float* steps;  // kEnds: sum of the steps [B][segments][D]
    ScanPlan plan;
};

// SW waves share a tile's states, SP each (more than 16 states: two or four).  Alone, a wave keeps all it knows of a position in
// registers; together they share the positions (sw, sw + SW, ... are this wave's: it computes their steps and finishes their outputs) and
// meet in LDS.
template <typename T, int SP, int SW, int MODE, bool GATED, bool FLAT>
__global__ __launch_bounds__(256, SP <= 8 ? 3 : 2) void scan_kernel(ScanRun r) {
    constexpr int kSet = kP * 2 * SP, kBc = FLAT ? 2 * kSet + 4 : kSet;  // FLAT: the second group's vectors, four banks on
    extern __shared__ float lds[];  // [waves][kBc]; SW > 1: then steps and step x [2][kP][64], sums over the states [SW][kP][64]
    constexpr int P = kP / SW;
    const ScanIn& in = r.in;
    const int lane = threadIdx.x & 63, tiles = r.plan.all_tiles;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned at_work = SW > 1 ? blockIdx.x : blockIdx.x * (blockDim.x >> 6) + wave, which = at_work / tiles;
    const int tile = at_work - which * tiles, sw = SW > 1 ? wave : 0, s0 = sw * SP;
    float* bc = lds + wave * kBc;
    float* shared = lds + SW * kBc + lane;
    float* sums = shared + 2 * kP * 64;
    int b = which / r.plan.segments;
    const int seg = which - b * r.plan.segments;
    // Whole sequences, as many waves as there is room for at once: long ones first, then the short ones from the shortest on, so that a
    // SIMD's waves are about as long together everywhere.
    if (r.plan.segments == 1) b = ranked(in.lengths, in.B, in.N, b < (in.B + 1) / 2 ? b : in.B - 1 - (b - (in.B + 1) / 2), lane);
    const int width = in.D_ / in.G, group = FLAT ? tile * 64 / width : tile / r.plan.tiles;
    const int first = FLAT ? 0 : group * width, wide = FLAT ? in.D_ : width;  // the channels that the tiles are cut from
    const int c0 = (FLAT ? tile : tile - group * r.plan.tiles) * 64 + lane;
    const bool is = c0 < wide;
    const int d = first + (is ? c0 : wide - 1);
    const int next_group = group + 1 < in.G ? group + 1 : group;
    const f32x4* bc4 = reinterpret_cast<const f32x4*>(bc + (FLAT && d / width != group ? kSet + 4 : 0));
    const int len = clamp_length(in.lengths, b, in.N), begin = seg * r.plan.seg_len;
    const int stop = segment_stop(r.plan, begin, in.N), end = stop < len ? stop : len;
    const unsigned bytes = static_cast<unsigned>(d) * sizeof(T);
    T* out = MODE & kOut ? static_cast<T*>(r.out) + static_cast<int64_t>(b) * in.N * in.D_ : nullptr;
    const float skip = in.D ? in.D[d] : 0.0f, bias = in.dt_bias ? in.dt_bias[d] : 0.0f;

    float h[SP], A[SP], total = 0.0f;
#pragma unroll
    for (int s = 0; s < SP; ++s) {
        A[s] = base2(in.A[static_cast<int64_t>(d) * in.S + state_at(s0 + s, in.S)]);
        h[s] = 0.0f;
    }
    if (!(MODE & kEnds)) {
        if (r.plan.segments > 1) {
            const int64_t from = static_cast<int64_t>(b) * r.plan.segments + seg;
#pragma unroll
            for (int s = 0; s < SP; ++s) {
                const int k = state_at(s0 + s, in.S);
                h[s] = r.ends[quad_at(from, in.S, in.D_, k / 4, d) + k % 4];
            }
        } else if (r.state) {
#pragma unroll
            for (int s = 0; s < SP; ++s) h[s] = r.state[(static_cast<int64_t>(b) * in.D_ + d) * in.S + state_at(s0 + s, in.S)];
        }
    }

    if (begin < end) {
        T xr[P], tr[P], zr[P];
        GroupVectors<T, SP> gv, gv2;  // (FLAT: and of the next group)
        const T *px = at<T>(in.x, b, begin + sw), *pt = at<T>(in.dt, b, begin + sw), *pz = at<T>(in.z, b, begin + sw);
        const auto fetch_whole = [&](int ahead) {
            px += ahead * kP * in.x.row;
            pt += ahead * kP * in.dt.row;
            pz += ahead * kP * in.z.row;
            gv.next(in, ahead);
            if (FLAT) gv2.next(in, ahead);
            load_whole<T, P>(px, SW * in.x.row, bytes, xr);
            load_whole<T, P>(pt, SW * in.dt.row, bytes, tr);
            if (GATED) load_whole<T, P>(pz, SW * in.z.row, bytes, zr);
        };
        float step[kP], put[kP], x[P], z[P];  // (SW > 1: step and put are in LDS)
        const auto settle = [&](auto whole, int l0) {  // what fetch has brought
            constexpr bool WHOLE = decltype(whole)::value;
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const int i = sw + k * SW;
                const bool on = WHOLE || l0 + i < end;
                const float st = on ? softplus(widen(tr[k]) + bias).value : 0.0f;
                x[k] = on ? widen(xr[k]) : 0.0f;
                if (GATED) z[k] = widen(zr[k]);
                if constexpr (SW > 1) {
                    shared[i * 64] = st;
                    shared[(kP + i) * 64] = st * x[k];
                } else {
                    step[k] = st;
                    put[k] = st * x[k];
                }
            }
            wave_sync();
            gv.template put<WHOLE>(bc, l0, len, lane);
            if (FLAT) gv2.template put<WHOLE>(bc + kSet + 4, l0, len, lane);
            wave_sync();
        };
        const auto block = [&](auto whole, int l0) {
            constexpr bool WHOLE = decltype(whole)::value;
            if (MODE & kSave) {
                float* place = r.saved + quad_at(static_cast<int64_t>(b) * ((in.N + kP - 1) / kP) + l0 / kP, in.S, in.D_, 0, 0);
#pragma unroll
                for (int q = 0; q < SP / 4; ++q)
                    *reinterpret_cast<f32x4*>(reinterpret_cast<char*>(place) + quad_bytes(in.D_, s0 / 4 + q, d)) = f32x4{h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]};
            }
            // The next block, or behind the last whole one that one again: without a branch nothing has to wait for it here.
            if (WHOLE) fetch_whole(l0 + 2 * kP <= end);
            constexpr int Q = SP / 4, R = MODE & kOut ? 2 * Q : Q;
            f32x4 v[2][R];  // Bm and Cm of a position; the next one's are read while this one's are used
#pragma unroll
            for (int q = 0; q < R; ++q) v[0][q] = bc4[q];
            float o[P];
#pragma unroll
            for (int i = 0; i < kP; ++i) {
                if (i + 1 < kP) {
#pragma unroll
                    for (int q = 0; q < R; ++q) v[(i + 1) & 1][q] = bc4[(i + 1) * 2 * Q + q];
                }
                __builtin_amdgcn_sched_barrier(0);
                const float step_i = SW > 1 ? shared[i * 64] : step[i], put_i = SW > 1 ? shared[(kP + i) * 64] : put[i];
                const f32x4(&now)[R] = v[i & 1];
                float y0 = 0.0f, y1 = 0.0f;
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    const f32x4 Bq = now[q];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int s = 4 * q + j;
                        h[s] = fmaf(exp2_fast(step_i * A[s]), h[s], put_i * Bq[j]);
                    }
                    if constexpr ((MODE & kOut) != 0) {
                        const f32x4 Cq = now[Q + q];
                        y0 = fmaf(h[4 * q], Cq[0], y0);
                        y1 = fmaf(h[4 * q + 1], Cq[1], y1);
                        y0 = fmaf(h[4 * q + 2], Cq[2], y0);
                        y1 = fmaf(h[4 * q + 3], Cq[3], y1);
                    }
                }
                if (MODE & kEnds) total += step_i;
                if constexpr ((MODE & kOut) != 0 && SW > 1) {
                    sums[(sw * kP + i) * 64] = y0 + y1;
                } else if constexpr ((MODE & kOut) != 0) {
                    const float y = fmaf(skip, x[i], y0 + y1);
                    o[i] = GATED ? y * silu(z[i]) : y;
                    asm volatile("" : "+v"(o[i]));  // computed here: moved behind a store's condition, it would keep the states of all eight positions
                }
            }
            if constexpr (SW > 1) {
                __syncthreads();
                if (MODE & kOut) {
#pragma unroll
                    for (int k = 0; k < P; ++k) {
                        float y = 0.0f;
#pragma unroll
                        for (int w = 0; w < SW; ++w) y += sums[(w * kP + sw + k * SW) * 64];
                        y = fmaf(skip, x[k], y);
                        o[k] = GATED ? y * silu(z[k]) : y;
                    }
                }
            }
            if (WHOLE) settle(std::true_type{}, l0 + kP);
            if (MODE & kOut) {
                T* to = out + static_cast<int64_t>(l0 + sw) * in.D_;
                unsigned at = bytes;
                asm volatile("" : "+v"(at));
#pragma unroll
                for (int k = 0; k < P; ++k, to += SW * in.D_)
                    if (WHOLE || l0 + sw + k * SW < end) give(to, at, o[k]);
            }
            if (SW > 1) __syncthreads();  // steps are there for the other waves, sums are free
        };
        gv.place(in, b, begin, group, s0, lane);
        if (FLAT) gv2.place(in, b, begin, next_group, s0, lane);
        int l0 = begin;
        if (begin + kP <= end) {
            fetch_whole(0);
            settle(std::true_type{}, begin);
            if (SW > 1) __syncthreads();
            for (; l0 + kP <= end; l0 += kP) block(std::true_type{}, l0);
        }
        if (l0 < end) {
            gv.place(in, b, l0, group, s0, lane);
            gv.load(in, l0, len);
            if (FLAT) {
                gv2.place(in, b, l0, next_group, s0, lane);
                gv2.load(in, l0, len);
            }
            load_rows<T, P>(in.x, b, l0 + sw, SW, len, bytes, xr);
            load_rows<T, P>(in.dt, b, l0 + sw, SW, len, bytes, tr);
            if (GATED) load_rows<T, P>(in.z, b, l0 + sw, SW, len, bytes, zr);
            settle(std::false_type{}, l0);
            if (SW > 1) __syncthreads();
            block(std::false_type{}, l0);
        }
    }
    if (MODE & kOut)
        for (int l = begin < end ? end : begin; l < stop; ++l)
            if (is && sw == 0) give(out + static_cast<int64_t>(l) * in.D_, bytes, 0.0f);
    if (MODE & kEnds) {
        const int64_t to = static_cast<int64_t>(b) * r.plan.segments + seg;
        if (is) {
#pragma unroll
            for (int s = 0; s < SP; ++s)
                if (s0 + s < in.S) r.ends[quad_at(to, in.S, in.D_, (s0 + s) / 4, d) + s % 4] = h[s];
            if (sw == 0) r.steps[to * in.D_ + d] = total;
        }
    } else if (r.final_state && is && (end == len && (begin < len || seg == 0))) {
#pragma unroll
        for (int s = 0; s < SP; ++s)
            if (s0 + s < in.S) r.final_state[(static_cast<int64_t>(b) * in.D_ + d) * in.S + s0 + s] = h[s];
    }
}

// A thread has four states of a channel and goes from segment to segment.  There are few of them, so workgroups are small: every compute
// unit has its own way to memory (56 segments of B=4 D=514 S=16: 8 us, in workgroups of 256 14).
constexpr int kJoin = 64;
template <bool BACK>
__global__ __launch_bounds__(kJoin) void join_segments_kernel(ScanIn in, ScanPlan p, const float* __restrict__ state, float* __restrict__ ends,
                                                            const float* __restrict__ steps) {
    const int64_t id = static_cast<int64_t>(blockIdx.x) * kJoin + threadIdx.x;
    const int64_t rest = id / in.D_;
    const int d = static_cast<int>(id - rest * in.D_), q = static_cast<int>(rest % quads(in.S));
    const int64_t b = rest / quads(in.S);
    if (b >= in.B) return;
    float A[4], h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int s = 4 * q + j;
        A[j] = s < in.S ? base2(in.A[static_cast<int64_t>(d) * in.S + s]) : 0.0f;
        h[j] = state && s < in.S ? state[(b * in.D_ + d) * in.S + s] : 0.0f;
    }
    // From the first segment on, or from the last: places and strides of `ends` and `steps`.
    const int64_t first = b * p.segments + (BACK ? p.segments - 1 : 0);
    const int64_t e_stride = (BACK ? -4 : 4) * static_cast<int64_t>(quads(in.S)) * in.D_, t_stride = BACK ? -in.D_ : in.D_;
    float* e = ends + quad_at(first, in.S, in.D_, q, d);
    const float* t = steps + first * in.D_ + d;
    const auto some = [&](auto many) {  // that many segments, their loads in flight together: the way along them is all waiting
        constexpr int U = decltype(many)::value;
        f32x4 made[U];
        float step[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            made[u] = *reinterpret_cast<const f32x4*>(e + u * e_stride);
            step[u] = t[u * t_stride];
        }
        const auto along = [&](auto careful) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                *reinterpret_cast<f32x4*>(e + u * e_stride) = f32x4{h[0], h[1], h[2], h[3]};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float power = step[u] * A[j], made_j = 4 * q + j < in.S ? made[u][j] : 0.0f;
                    const bool stays = decltype(careful)::value && __builtin_isinf(h[j]) && __builtin_isfinite(power);
                    h[j] = stays ? h[j] + made_j : fmaf(exp2_fast(power), h[j], made_j);
                }
            }
        };
        // The decays of a segment together may be below every float where each by itself is not, and make NaN of an infinite state that
        // stays one.  Where there is a NaN at the end, the same segments once more with a look at that.
        const float h0[4] = {h[0], h[1], h[2], h[3]};
        along(std::false_type{});
        if (__builtin_isnan(h[0] + h[1] + h[2] + h[3])) {
#pragma unroll
            for (int j = 0; j < 4; ++j) h[j] = h0[j];
            along(std::true_type{});
        }
        e += U * e_stride;
        t += U * t_stride;
    };
    int k = 0;
    for (; k + 16 <= p.segments; k += 16) some(std::integral_constant<int, 16>{});
    for (; k + 4 <= p.segments; k += 4) some(std::integral_constant<int, 4>{});
    for (; k < p.segments; ++k) some(std::integral_constant<int, 1>{});
}

// ---- one position ---------------------------------------------------------------------------------------------
// A thread has four states of a channel and `many` streams one after the other, their states in flight together; LQ threads a
// channel.  The states read and written are what bounds it: 512 streams of D=2048 S=16, 143 MB, 25.0 us (5.7 TB/s: a part of them stays in
// the memory-side cache); four of D=1024 3.2 us, bound by one pass's latency.
template <typename T, int LQ, int MANY, bool WHOLE>
__global__ __launch_bounds__(256) void step_kernel(ScanIn in, float* __restrict__ state, T* __restrict__ out) {
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t ch = id / LQ, row = ch / in.D_;
    const int q = threadIdx.x % LQ, d = static_cast<int>(ch - row * in.D_), s0 = 4 * q;
    const int b0 = static_cast<int>(row) * MANY;
    if (row * MANY >= in.B) return;  // whole groups of LQ threads leave together
    const int group = d / (in.D_ / in.G);
    const float skip = in.D ? in.D[d] : 0.0f, bias = in.dt_bias ? in.dt_bias[d] : 0.0f;
    float A[4], h[MANY][4];
    T xr[MANY], tr[MANY], zr[MANY], Br[MANY][4], Cr[MANY][4];
#pragma unroll
    for (int m = 0; m < MANY; ++m) {
        const int b = b0 + m < in.B ? b0 + m : in.B - 1;
        const float* mine = state + (static_cast<int64_t>(b) * in.D_ + d) * in.S + s0;
        if (WHOLE) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(mine);
#pragma unroll
            for (int j = 0; j < 4; ++j) h[m][j] = v[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) h[m][j] = s0 + j < in.S ? mine[j] : 0.0f;
        }
        xr[m] = at<T>(in.x, b, 0)[d];
        tr[m] = at<T>(in.dt, b, 0)[d];
        if (in.z.data) zr[m] = at<T>(in.z, b, 0)[d];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int s = WHOLE || s0 + j < in.S ? s0 + j : 0;
            Br[m][j] = (at<T>(in.Bm, b, 0) + group * in.b_group)[s];
            Cr[m][j] = (at<T>(in.Cm, b, 0) + group * in.c_group)[s];
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) A[j] = WHOLE || s0 + j < in.S ? base2(in.A[static_cast<int64_t>(d) * in.S + s0 + j]) : 0.0f;
#pragma unroll
    for (int m = 0; m < MANY; ++m) {
        const float step = softplus(widen(tr[m]) + bias).value, x = widen(xr[m]), put = step * x;
        float y = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            h[m][j] = fmaf(exp2_fast(step * A[j]), h[m][j], put * widen(Br[m][j]));
            y = WHOLE || s0 + j < in.S ? fmaf(h[m][j], widen(Cr[m][j]), y) : y;
        }
#pragma unroll
        for (int k = 1; k < LQ; k *= 2) y += __shfl_xor(y, k);
        y = fmaf(skip, x, y);
        if (in.z.data) y *= silu(widen(zr[m]));
        if (b0 + m < in.B) {
            float* mine = state + (static_cast<int64_t>(b0 + m) * in.D_ + d) * in.S + s0;
            if (WHOLE) {
                *reinterpret_cast<f32x4*>(mine) = f32x4{h[m][0], h[m][1], h[m][2], h[m][3]};
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (s0 + j < in.S) mine[j] = h[m][j];
            }
            if (q == 0) put1(out + static_cast<int64_t>(b0 + m) * in.D_ + d, y);
        }
    }
}

template <typename T, int LQ>
hipError_t step_of(const ScanIn& in, float* state, void* out, hipStream_t st) {
    // four streams a thread once that leaves 2048 workgroups
    const bool many = static_cast<int64_t>(in.B) * in.D_ * LQ >= (int64_t{2048} * 256 * 4);
    const int M = many ? 4 : 1;
    const int64_t threads = static_cast<int64_t>((in.B + M - 1) / M) * in.D_ * LQ;
    if (!fits((threads + 255) / 256, 256)) return hipErrorInvalidValue;
    const bool whole = in.S == 4 * LQ && (reinterpret_cast<uintptr_t>(state) & 15) == 0;
    const auto kernel = many ? (whole ? step_kernel<T, LQ, 4, true> : step_kernel<T, LQ, 4, false>)
                             : (whole ? step_kernel<T, LQ, 1, true> : step_kernel<T, LQ, 1, false>);
    kernel<<<static_cast<unsigned>((threads + 255) / 256), 256, 0, st>>>(in, state, static_cast<T*>(out));
    return hipGetLastError();
}

// ---- launches -------------------------------------------------------------------------------------------------

template <typename T, int SP, int SW, int MODE>
hipError_t scan_launch(const ScanRun& r, hipStream_t st) {
    const int64_t tiles = static_cast<int64_t>(r.plan.all_tiles) * r.in.B * r.plan.segments;
    constexpr bool kGate = (MODE & kOut) != 0, kFlat = SW == 1;
    const bool gated = kGate && r.in.z.data;
    const auto kernel = r.plan.flat ? (gated ? scan_kernel<T, SP, SW, MODE, kGate, kFlat> : scan_kernel<T, SP, SW, MODE, false, kFlat>)
                                    : (gated ? scan_kernel<T, SP, SW, MODE, kGate, false> : scan_kernel<T, SP, SW, MODE, false, false>);
    const int w = SW > 1 ? SW : waves_together(r.plan.all_tiles);
    const size_t bytes = sizeof(float) * (w * (r.plan.flat ? 2 * kP * 2 * SP + 4 : kP * 2 * SP) + (SW > 1 ? (2 + SW) * kP * 64 : 0));
    kernel<<<static_cast<unsigned>(tiles * SW / w), 64 * w, bytes, st>>>(r);
    return hipGetLastError();
}

template <typename T, int SP, int SW>
hipError_t scan_run(const ScanRun& r, hipStream_t st) {
    if (r.plan.segments > 1) {
        if (const hipError_t e = scan_launch<T, SP, SW, kEnds>(r, st); e != hipSuccess) return e;
        if (const hipError_t e = launch_join_segments(r.in, r.plan, r.state, r.ends, r.steps, false, st); e != hipSuccess) return e;
    }
    if (!r.out) return scan_launch<T, SP, SW, kSave>(r, st);
    return r.saved ? scan_launch<T, SP, SW, kOut | kSave>(r, st) : scan_launch<T, SP, SW, kOut>(r, st);
}

template <typename T>
hipError_t scan_of(const ScanRun& r, hipStream_t st) {
    if (r.in.S <= 4) return scan_run<T, 4, 1>(r, st);
    if (r.in.S <= 8) return scan_run<T, 8, 1>(r, st);
    if (r.in.S <= 16) return scan_run<T, 16, 1>(r, st);
    return r.in.S <= 32 ? scan_run<T, 16, 2>(r, st) : scan_run<T, 16, 4>(r, st);
}

size_t ends_bytes(const ScanPlan& p, int B, int D, int S) {
    return up256(static_cast<size_t>(B) * p.segments * quads(S) * D * 16);
}

}  // namespace

hipError_t launch_join_segments(const ScanIn& in, const ScanPlan& p, const float* state, float* ends, const float* steps, bool back, hipStream_t st) {
    const int64_t threads = static_cast<int64_t>(in.B) * in.D_ * quads(in.S);
    const unsigned blocks = static_cast<unsigned>((threads + kJoin - 1) / kJoin);
    if (back) join_segments_kernel<true><<<blocks, kJoin, 0, st>>>(in, p, state, ends, steps);
    else join_segments_kernel<false><<<blocks, kJoin, 0, st>>>(in, p, state, ends, steps);
    return hipGetLastError();
}

size_t scan_saved_bytes(int B, int N, int D, int S) { return up256(static_cast<size_t>(B) * scan_blocks(N) * quads(S) * D * 16); }

size_t scan_workspace(int B, int N, int D, int S, int G) {
    const ScanPlan p = forward_plan(B, N, D, S, G);
    if (p.segments == 1) return 256;
    return ends_bytes(p, B, D, S) + up256(static_cast<size_t>(B) * p.segments * D * 4);
}

hipError_t run_state_scan(int dtype, const ScanIn& in, const float* state, void* out, float* final_state, float* saved, void* ws, hipStream_t st) {
    ScanRun r{in, state, out, final_state, saved, nullptr, nullptr, forward_plan(in.B, in.N, in.D_, in.S, in.G)};
    if (!scan_fits(in.B, in.N, in.D_, in.S, in.G, r.plan)) return hipErrorInvalidValue;
    if (r.plan.segments > 1) {
        r.ends = static_cast<float*>(ws);
        r.steps = reinterpret_cast<float*>(static_cast<char*>(ws) + ends_bytes(r.plan, in.B, in.D_, in.S));
    }
    return dtype ? scan_of<uint16_t>(r, st) : scan_of<float>(r, st);
}

hipError_t launch_state_scan(int dtype, const ScanIn& in, const float* state, void* out, float* final_state, void* saved, void* ws, hipStream_t st) {
    return run_state_scan(dtype, in, state, out, final_state, static_cast<float*>(saved), ws, st);
}

hipError_t launch_state_step(int dtype, const ScanIn& in, float* state, void* out, hipStream_t st) {
    const int n = quads(in.S);
#define LCCRF_STEP(LQ) (dtype ? step_of<uint16_t, LQ>(in, state, out, st) : step_of<float, LQ>(in, state, out, st))
    return n <= 1 ? LCCRF_STEP(1) : n <= 2 ? LCCRF_STEP(2) : n <= 4 ? LCCRF_STEP(4) : n <= 8 ? LCCRF_STEP(8) : LCCRF_STEP(16);
#undef LCCRF_STEP
}

}  // namespace enc
}  // namespace lccrf
