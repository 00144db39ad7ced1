// Gradient of the selective state space scan.
//
// With dh[l] = dy[l] Cm[l] + a[l+1] dh[l+1] running backwards,
//     dCm = sum_channels dy h,   dBm = sum_channels dh put,   dput = sum_s dh Bm,   back = dh a h[l-1]  (by the decay's logarithm),
//     dx = dput step + D dy,     dv = (dput x + sum_s back A) sigmoid(v),    dA = sum_positions back step.
// (A state that is held several times has a share of Cm, so of dh and of what follows from it; dA, dBm and dstate, which look at one
// copy, take it times the copies.)
// The states in front of every eighth position are saved by the forward pass; eight positions are run again from there, their
// states kept in registers, and then gone through backwards.  27 vector instructions an update with 16 states (counted: 5 forwards, 10
// backwards, the rest for sums over the channels and what is computed once a channel), two of them exponentials: vector arithmetic
// bounds it (B=128 N=256 D=1024 S=16, bfloat16, ragged: 313 us, the vector pipes busy 96 % of them).
//
// A wave has 64 channels and up to 8 states: 72 registers of states, three waves a SIMD.  Measured on the whole training step of that
// batch: 16 states a wave spilled, and left no registers for the next positions' inputs (1290 us against 536 at that time); the
// decays kept as well would save the second exponential, but take 64 registers and with them the third wave (470 us against 448).
// More states are shared by several waves of a workgroup, which also share what is computed once a channel, and whose sums over
// the states meet in LDS.
// The sums over the channels are taken by halving: two registers and two halves of the wave become one register whose
// halves hold one sum each (a swap and an addition), and so on, 35 instructions for the 16 sums of a position; the waves of a
// workgroup meet in LDS, workgroups through memory, always in the same order.
#include "lccrf_state.h"

namespace lccrf {
namespace enc {
namespace {

struct GradPlan {
    ScanPlan scan;
    int state_waves;  // waves that share a channel's states: 1, 2, 4 or 8
    int tile_waves;   // tiles of 64 channels a workgroup
    int parts;        // workgroups a group's channels are spread over
};

GradPlan grad_plan(int B, int N, int D, int S, int G) {
    GradPlan p;
    p.state_waves = S <= 8 ? 1 : S <= 16 ? 2 : S <= 32 ? 4 : 8;
    p.scan = scan_plan(B, N, D, G, false, p.state_waves, 3 * 1024, 2);  // three waves a SIMD
    p.tile_waves = p.state_waves >= 4 ? 1 : 4 / p.state_waves;
    while (p.scan.tiles % p.tile_waves) p.tile_waves /= 2;  // no wave without a channel
    p.parts = p.scan.tiles / p.tile_waves;
    return p;
}

struct GradRun {
    ScanIn in;
    AnyRows dout;
    ScanGrads g;
    const float* saved;
    float* ends;     // segments > 1: the gradient by the state behind every segment
    float* steps;
    float* part_bc;  // parts > 1: [parts][2][B][N][G][S]
    float* part_a;   // [B * segments][D][S]
    float* part_d;   // [B * segments * state_waves][2][D]: dD, ddt_bias
    GradPlan plan;
};

template <int CTRL> __device__ __forceinline__ float from_lane(float x) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kRor8 = 0x128;

// Two sums in one register: lanes with the bit clear go on with x, the others with y.
template <int CTRL> __device__ __forceinline__ float halve(float x, float y, bool bit) {
    return (bit ? y : x) + from_lane<CTRL>(bit ? x : y);
}
__device__ __forceinline__ float halve32(float x, float y) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float halve16(float x, float y) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// The rest of the way for n = SP / 2 registers, each of which holds two sums of every half of the wave (halve32 of dBm and dCm of a
// state, halve16 of states s and s + n): lane k ends with sum k / (32 / SP) of (dBm of all states, dCm of all states).
template <int N> __device__ __forceinline__ float lane_sums(float (&v)[N], int lane) {
    static_assert(N == 2 || N == 4, "");
#pragma unroll
    for (int i = 0; i < N / 2; ++i) v[i] = halve<kRor8>(v[i], v[i + N / 2], lane & 8);
    if constexpr (N == 4) v[0] = halve<kHalfMirror>(v[0], v[1], lane & 4);
    else v[0] += from_lane<kHalfMirror>(v[0]);
    v[0] += from_lane<kXor2>(v[0]);
    return v[0] + from_lane<kXor1>(v[0]);
}

// A tile of fewer than 64 channels: lanes past them hold channels once more, m = 2^k times or 2m times in all, and count in the sums over
// the channels for 1/m or 1/(2m): what the copies add up to is exact, and infinite or NaN where the channel by itself is (a count of 0 would make
// NaN of an infinite one).
struct LaneShare { int channel; float share; };
__device__ __forceinline__ LaneShare lane_share(int channels, int lane) {
    if (channels >= 64) return {lane, 1.0f};
    int m = 1;
    while (2 * m * channels <= 64) m *= 2;
    const int more = 64 / m - channels;  // channels with 2m lanes: the first ones
    const int channel = lane < channels * m ? lane % channels : (lane - channels * m) % (more > 0 ? more : 1);
    return {channel, channel < more ? 0.5f / m : 1.0f / m};
}

// dy of a position: the gradient by y.
__device__ __forceinline__ float through_gate(float dout, float z, bool gated) { return gated ? dout * silu(z) : dout; }

// What a segment makes of 0 behind it, and the sum of its steps.
template <typename T, int SP>
__global__ __launch_bounds__(256, 2) void back_ends_kernel(GradRun r) {
    extern __shared__ float lds[];  // [waves][kP][2 * SP]
    const ScanIn& in = r.in;
    const ScanPlan& plan = r.plan.scan;
    const int lane = threadIdx.x & 63, tiles = in.G * plan.tiles;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned at_work = blockIdx.x * (blockDim.x >> 6) + wave, which = at_work / tiles;
    const int tile = at_work - which * tiles, s0 = blockIdx.y * SP;
    float* bc = lds + wave * (kP * 2 * SP);
    const int b = which / plan.segments, seg = which - b * plan.segments;
    const int width = in.D_ / in.G, group = tile / plan.tiles, c0 = (tile - group * plan.tiles) * 64 + lane;
    const bool is = c0 < width;
    const int d = group * width + (is ? c0 : width - 1);
    const int len = clamp_length(in.lengths, b, in.N), begin = seg * plan.seg_len;
    const int stop = segment_stop(plan, begin, in.N), end = stop < len ? stop : len;
    const bool gated = in.z.data != nullptr;
    const unsigned bytes = static_cast<unsigned>(d) * sizeof(T);
    const float bias = in.dt_bias ? in.dt_bias[d] : 0.0f;
    float dh[SP], A[SP], total = 0.0f;
#pragma unroll
    for (int s = 0; s < SP; ++s) {
        A[s] = base2(in.A[static_cast<int64_t>(d) * in.S + state_at(s0 + s, in.S)]);
        dh[s] = 0.0f;
    }
    if (begin < end) {
        T tr[kP], zr[kP], dr[kP];
        GroupVectors<T, SP> gv;
        const int last = begin + (end - begin - 1) / kP * kP;
        gv.place(in, b, last, group, s0, lane);
        gv.load(in, last, len);
        load_rows<T, kP>(in.dt, b, last, 1, len, bytes, tr);
        load_rows<T, kP>(r.dout, b, last, 1, len, bytes, dr);
        if (gated) load_rows<T, kP>(in.z, b, last, 1, len, bytes, zr);
        const T *pt = at<T>(in.dt, b, last), *pd = at<T>(r.dout, b, last), *pz = at<T>(in.z, b, last);
        for (int l0 = last; l0 >= begin; l0 -= kP) {
            float step[kP], dy[kP];
#pragma unroll
            for (int i = 0; i < kP; ++i) {
                const bool on = l0 + i < end;
                step[i] = on ? softplus(widen(tr[i]) + bias).value : 0.0f;
                dy[i] = on ? through_gate(widen(dr[i]), gated ? widen(zr[i]) : 0.0f, gated) : 0.0f;
                total += step[i];
            }
            wave_sync();
            gv.template put<false>(bc, l0, len, lane);
            wave_sync();
            if (l0 > begin) {
                pt -= kP * in.dt.row;
                pd -= kP * r.dout.row;
                pz -= kP * in.z.row;
                gv.next(in, -1);
                load_whole<T, kP>(pt, in.dt.row, bytes, tr);
                load_whole<T, kP>(pd, r.dout.row, bytes, dr);
                if (gated) load_whole<T, kP>(pz, in.z.row, bytes, zr);
            }
#pragma unroll
            for (int i = kP - 1; i >= 0; --i) {
                const f32x4* C4 = reinterpret_cast<const f32x4*>(bc + i * 2 * SP + SP);
#pragma unroll
                for (int q = 0; q < SP / 4; ++q) {
                    const f32x4 Cq = C4[q];
#pragma unroll
                    for (int j = 0; j < 4; ++j) dh[4 * q + j] = exp2_fast(step[i] * A[4 * q + j]) * fmaf(dy[i], Cq[j], dh[4 * q + j]);
                }
            }
        }
    }
    const int64_t to = static_cast<int64_t>(b) * plan.segments + seg;
    if (is) {
#pragma unroll
        for (int s = 0; s < SP; ++s)
            if (s0 + s < in.S) r.ends[quad_at(to, in.S, in.D_, (s0 + s) / 4, d) + s % 4] = dh[s];
        if (s0 == 0) r.steps[to * in.D_ + d] = total;
    }
}

// Values of a channel and position that all waves of a tile need, in LDS: [kScal][kP][64] a tile.
enum { kStep, kDy, kX, kSlope, kDz, kScal };

// Floats of LDS: Bm and Cm a wave, `scal` a tile, the sums over the states (y, dput, sum back A) a wave, the sums over the channels a wave.
template <int SP, int SW> __host__ __device__ constexpr int grad_lds(int tile_waves) {
    return tile_waves * (SW * (kP * 2 * SP) + kScal * kP * 64 + SW * (3 * kP * 64) + SW * (kP * 2 * SP));
}

template <typename T, int SP, int SW, bool GATED>
__global__ __launch_bounds__(SW == 8 ? 512 : 256, SP == 4 ? 4 : SW == 1 ? 2 : 3) void scan_grad_kernel(GradRun r) {
    extern __shared__ float lds[];
    constexpr int P = kP / SW;  // positions whose values of a channel this wave computes: sw, sw + SW, ...
    const ScanIn& in = r.in;
    const ScanPlan& plan = r.plan.scan;
    const int CT = r.plan.tile_waves, waves = SW * CT;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int sw = wave % SW, ct = wave / SW, s0 = sw * SP;
    unsigned which = blockIdx.x / r.plan.parts;
    const int part = blockIdx.x - which * r.plan.parts;
    const unsigned bs = which / in.G;
    const int group = which - bs * in.G;
    int b = bs / plan.segments;
    const int seg = bs - b * plan.segments;
    if (plan.segments == 1) b = ranked(in.lengths, in.B, in.N, b, lane);
    const int tile = part * CT + ct, width = in.D_ / in.G;
    const LaneShare held = lane_share(width - tile * 64, lane);
    const bool is = lane < width - tile * 64, full_tile = tile * 64 + 64 <= width;
    const int d = group * width + tile * 64 + held.channel;
    const int len = clamp_length(in.lengths, b, in.N), begin = seg * plan.seg_len;
    const int stop = segment_stop(plan, begin, in.N), end = stop < len ? stop : len;
    const int64_t from = static_cast<int64_t>(b) * plan.segments + seg;

    float* bc = lds + wave * (kP * 2 * SP);
    float* scal = lds + waves * (kP * 2 * SP) + ct * (kScal * kP * 64) + lane;
    float* sums = lds + waves * (kP * 2 * SP) + CT * (kScal * kP * 64) + ct * SW * (3 * kP * 64) + lane;  // of this tile: [SW][3][kP][64]
    float* my_sums = sums + sw * (3 * kP * 64);
    float* red = lds + waves * (kP * 2 * SP) + CT * (kScal * kP * 64) + waves * (3 * kP * 64);            // [waves][kP][2 * SP]

    const float skip = in.D ? in.D[d] : 0.0f, bias = in.dt_bias ? in.dt_bias[d] : 0.0f;
    const int64_t row = static_cast<int64_t>(b) * in.N;
    const unsigned bytes = static_cast<unsigned>(d) * sizeof(T);
    T* dx = static_cast<T*>(r.g.dx) + row * in.D_;
    T* ddt = static_cast<T*>(r.g.ddt) + row * in.D_;
    T* dz = static_cast<T*>(r.g.dz) + row * in.D_;
    float dh[SP], A[SP], dA[SP], sum_dD = 0.0f, sum_dv = 0.0f;
#pragma unroll
    for (int s = 0; s < SP; ++s) {
        A[s] = base2(in.A[static_cast<int64_t>(d) * in.S + state_at(s0 + s, in.S)]);
        dh[s] = 0.0f;
        dA[s] = 0.0f;
    }
    if (plan.segments > 1) {
#pragma unroll
        for (int s = 0; s < SP; ++s) {
            const int k = state_at(s0 + s, in.S);
            dh[s] = r.ends[quad_at(from, in.S, in.D_, k / 4, d) + k % 4];
        }
    }

    if (begin < end) {
        T xr[P], tr[P], zr[P], dr[P];
        f32x4 before[SP / 4];
        GroupVectors<T, SP> gv;
        const int last = begin + (end - begin - 1) / kP * kP;
        const int64_t block = static_cast<int64_t>(in.D_) * quads(in.S) * 4;
        const float* ps = r.saved + (static_cast<int64_t>(b) * ((in.N + kP - 1) / kP) + last / kP) * block;
        const unsigned quad = quad_bytes(in.D_, s0 / 4, d);
        const auto load_before = [&] {
#pragma unroll
            for (int q = 0; q < SP / 4; ++q)
                before[q] = *reinterpret_cast<const f32x4*>(reinterpret_cast<const char*>(ps) + (quad + static_cast<unsigned>(q * in.D_) * 16));
        };
        load_before();
        gv.place(in, b, last, group, s0, lane);
        gv.load(in, last, len);
        load_rows<T, P>(in.x, b, last + sw, SW, len, bytes, xr);
        load_rows<T, P>(in.dt, b, last + sw, SW, len, bytes, tr);
        load_rows<T, P>(r.dout, b, last + sw, SW, len, bytes, dr);
        if (GATED) load_rows<T, P>(in.z, b, last + sw, SW, len, bytes, zr);
        const T *px = at<T>(in.x, b, last + sw), *pt = at<T>(in.dt, b, last + sw), *pd = at<T>(r.dout, b, last + sw), *pz = at<T>(in.z, b, last + sw);
        const auto fetch = [&] {  // the block in front
            ps -= block;
            px -= kP * in.x.row;
            pt -= kP * in.dt.row;
            pd -= kP * r.dout.row;
            pz -= kP * in.z.row;
            load_before();
            gv.next(in, -1);
            load_whole<T, P>(px, SW * in.x.row, bytes, xr);
            load_whole<T, P>(pt, SW * in.dt.row, bytes, tr);
            load_whole<T, P>(pd, SW * r.dout.row, bytes, dr);
            if (GATED) load_whole<T, P>(pz, SW * in.z.row, bytes, zr);
        };
        const auto eight = [&](auto whole, int l0) {
            constexpr bool WHOLE = decltype(whole)::value;
            float h[kP + 1][SP];  // h[i]: in front of position i
#pragma unroll
            for (int s = 0; s < SP; ++s) h[0][s] = before[s / 4][s % 4];
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const int i = sw + k * SW;
                const bool on = WHOLE || l0 + i < end;
                const Softplus sp = softplus(widen(tr[k]) + bias);
                const float x = widen(xr[k]), dout = widen(dr[k]), z = GATED ? widen(zr[k]) : 0.0f, gate = sigmoid(z);
                float* to = scal + i * 64;
                to[kStep * kP * 64] = on ? sp.value : 0.0f;
                to[kDy * kP * 64] = on ? (GATED ? dout * (z * gate) : dout) : 0.0f;
                to[kX * kP * 64] = on ? x : 0.0f;
                to[kSlope * kP * 64] = sp.slope;
                if (GATED) to[kDz * kP * 64] = dout * gate * fmaf(z, 1.0f - gate, 1.0f);
            }
            gv.template put<WHOLE>(bc, l0, len, lane);
            if (SW > 1) __syncthreads();
            else wave_sync();
            // forwards
#pragma unroll
            for (int i = 0; i < kP; ++i) {
                const f32x4* B4 = reinterpret_cast<const f32x4*>(bc + i * 2 * SP);
                const float step = scal[(kStep * kP + i) * 64], put = step * scal[(kX * kP + i) * 64];
                float y0 = 0.0f, y1 = 0.0f;
#pragma unroll
                for (int q = 0; q < SP / 4; ++q) {
                    const f32x4 Bq = B4[q];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int s = 4 * q + j;
                        h[i + 1][s] = fmaf(exp2_fast(step * A[s]), h[i][s], put * Bq[j]);
                    }
                    if (GATED) {  // y itself is what dz needs
                        const f32x4 Cq = B4[SP / 4 + q];
                        y0 = fmaf(h[i + 1][4 * q], Cq[0], y0);
                        y1 = fmaf(h[i + 1][4 * q + 1], Cq[1], y1);
                        y0 = fmaf(h[i + 1][4 * q + 2], Cq[2], y0);
                        y1 = fmaf(h[i + 1][4 * q + 3], Cq[3], y1);
                    }
                }
                if (GATED) my_sums[i * 64] = y0 + y1;
            }
            // backwards
#pragma unroll
            for (int i = kP - 1; i >= 0; --i) {
                const f32x4* B4 = reinterpret_cast<const f32x4*>(bc + i * 2 * SP);
                const float step = scal[(kStep * kP + i) * 64], put = step * scal[(kX * kP + i) * 64], dy = scal[(kDy * kP + i) * 64];
                float v[SP / 2], dput0 = 0.0f, dput1 = 0.0f, back0 = 0.0f, back1 = 0.0f, own_put = put, own_dy = dy;
                if (!full_tile) {
                    own_put = put * held.share;
                    own_dy = dy * held.share;
                }
                const auto one = [&](int s, float Bs, float Cs, float& dput, float& sum) {
                    const float e = fmaf(dy, Cs, dh[s]);
                    dh[s] = e * exp2_fast(step * A[s]);
                    // (past the end dh is 0, but the last state, which no decay works on, may be infinite)
                    const float back = WHOLE || l0 + i < end ? dh[s] * h[i][s] : 0.0f;
                    dput = fmaf(e, Bs, dput);
                    sum = fmaf(back, A[s], sum);
                    dA[s] = fmaf(back, step, dA[s]);
                    asm volatile("" : "+v"(dA[s]));  // here: gathered behind the loop it would keep `back` of all eight positions
                    return halve32(e * own_put, own_dy * h[i + 1][s]);
                };
                // states s and s + SP / 2 together, so that few sums are under way at a time
                const f32x4 B1 = B4[0], C1 = B4[SP / 4], B2 = B4[SP / 4 - 1], C2 = B4[SP / 2 - 1];
#pragma unroll
                for (int s = 0; s < SP / 2; ++s) {
                    const int k = SP == 4 ? s + 2 : s;
                    const float first = one(s, B1[s], C1[s], dput0, back0);
                    v[s] = halve16(first, one(s + SP / 2, B2[k], C2[k], dput1, back1));
                }
                my_sums[(kP + i) * 64] = dput0 + dput1;
                my_sums[(2 * kP + i) * 64] = (back0 + back1) * kLn2f;
                const float sum = lane_sums<SP / 2>(v, lane);
                if (lane % (32 / SP) == 0) red[(wave * kP + i) * (2 * SP) + lane / (32 / SP)] = sum;
                if (i == kP / 2 && l0 > begin) fetch();  // into the registers of the positions that are done
            }
            __syncthreads();
            const int64_t first = static_cast<int64_t>(l0 + sw) * in.D_;
            T *tx = dx + first, *tt = ddt + first, *tz = dz + first;
            unsigned o = bytes;
            asm volatile("" : "+v"(o));
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const int i = sw + k * SW;
                float y = 0.0f, dput = 0.0f, back = 0.0f;
#pragma unroll
                for (int w = 0; w < SW; ++w) {
                    if (GATED) y += sums[(w * 3 * kP + i) * 64];
                    dput += sums[(w * 3 * kP + kP + i) * 64];
                    back += sums[(w * 3 * kP + 2 * kP + i) * 64];
                }
                const float* own = scal + i * 64;
                const float step = own[kStep * kP * 64], dy = own[kDy * kP * 64], x = own[kX * kP * 64];
                const float dv = fmaf(dput, x, back) * own[kSlope * kP * 64];
                if (WHOLE || l0 + i < end) {
                    sum_dv += dv;
                    sum_dD = fmaf(dy, x, sum_dD);
                    give(tx, o, fmaf(dput, step, skip * dy));
                    give(tt, o, dv);
                    if (GATED) give(tz, o, own[kDz * kP * 64] * fmaf(skip, x, y));
                }
                tx += SW * in.D_;
                tt += SW * in.D_;
                tz += SW * in.D_;
            }
            // The sums over the channels: position i, Bm or Cm, state s, from the waves of all tiles.
            const int64_t group_row = (row + l0) * in.G * in.S;
            unsigned k = threadIdx.x;
            asm volatile("" : "+v"(k));  // what follows from it is a few shifts: not worth registers through the loop
            for (; k < kP * SW * 2 * SP; k += 64 * waves) {
                const int i = k / (SW * 2 * SP), s = k % (SW * SP);
                const bool c = k / (SW * SP) & 1;
                if ((WHOLE || l0 + i < end) && s < in.S) {
                    const float* from = red + (s / SP * kP + i) * (2 * SP) + c * SP + s % SP;
                    float sum = from[0];
                    for (int t = 1; t < CT; ++t) sum += from[t * (SW * kP * 2 * SP)];
                    if (!c) sum *= copies_of(s, in.S);
                    const int to = (i * in.G + group) * in.S + s;
                    if (r.plan.parts == 1) put1((c ? static_cast<T*>(r.g.dCm) : static_cast<T*>(r.g.dBm)) + group_row + to, sum);
                    else (r.part_bc + (static_cast<int64_t>(part) * 2 + c) * in.B * in.N * in.G * in.S + group_row)[to] = sum;
                }
            }
            // `sums` and `red` are next written behind the next barrier, of the next eight positions (SW = 1 has none there)
            if (SW == 1) __syncthreads();
        };
        int l0 = last;
        if (l0 + kP > end) {
            eight(std::false_type{}, l0);
            l0 -= kP;
        }
        for (; l0 >= begin; l0 -= kP) eight(std::true_type{}, l0);
    }
    // Positions past the end.
    for (int l = begin < end ? end : begin; l < stop; ++l) {
        const int64_t to = static_cast<int64_t>(l) * in.D_;
        if (is && sw == 0) {
            give(dx + to, bytes, 0.0f);
            give(ddt + to, bytes, 0.0f);
            if (GATED) give(dz + to, bytes, 0.0f);
        }
        if (r.plan.parts == 1)
            for (int s = threadIdx.x; s < in.S; s += blockDim.x) {
                put1(static_cast<T*>(r.g.dBm) + ((row + l) * in.G + group) * in.S + s, 0.0f);
                put1(static_cast<T*>(r.g.dCm) + ((row + l) * in.G + group) * in.S + s, 0.0f);
            }
    }
    if (is) {
#pragma unroll
        for (int s = 0; s < SP; ++s)
            if (s0 + s < in.S) r.part_a[(from * in.D_ + d) * in.S + s0 + s] = dA[s] * copies_of(s0 + s, in.S);
        float* pd = r.part_d + (from * SW + sw) * 2 * in.D_ + d;
        pd[0] = sum_dD;
        pd[in.D_] = sum_dv;
        if (r.g.dstate && seg == 0) {
#pragma unroll
            for (int s = 0; s < SP; ++s)
                if (s0 + s < in.S) r.g.dstate[(static_cast<int64_t>(b) * in.D_ + d) * in.S + s0 + s] = dh[s] * copies_of(s0 + s, in.S);
        }
    }
}

// dBm and dCm from the workgroups that share a group; 0 past the end.  A read of their partial sums (B=128 N=256 D=1024 S=16: 8 us).
template <typename T>
__global__ __launch_bounds__(256) void group_sums_kernel(GradRun r) {
    const ScanIn& in = r.in;
    const int64_t all = static_cast<int64_t>(in.B) * in.N * in.G * in.S, id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (id >= all) return;
    const int64_t pos = id / (in.G * in.S);
    const int b = static_cast<int>(pos / in.N), l = static_cast<int>(pos - static_cast<int64_t>(b) * in.N);
    float sB = 0.0f, sC = 0.0f;
    if (l < clamp_length(in.lengths, b, in.N))
        for (int p = 0; p < r.plan.parts; ++p) {
            sB += r.part_bc[2 * p * all + id];
            sC += r.part_bc[(2 * p + 1) * all + id];
        }
    put1(static_cast<T*>(r.g.dBm) + id, sB);
    put1(static_cast<T*>(r.g.dCm) + id, sC);
}

// dA, dD and ddt_bias: columns summed over their rows, sixteen threads a column (the same batch: 5 us).
__global__ __launch_bounds__(1024) void column_sums_kernel(GradRun r, int a_blocks, int blocks) {
    __shared__ float sums[16][64];
    const ScanIn& in = r.in;
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
    for (int block = blockIdx.x; block < blocks; block += gridDim.x) {
        const bool isA = block < a_blocks;
        const int64_t columns = isA ? static_cast<int64_t>(in.D_) * in.S : 2 * static_cast<int64_t>(in.D_);
        const int64_t col = static_cast<int64_t>(isA ? block : block - a_blocks) * 64 + x;
        const int rows = in.B * r.plan.scan.segments * (isA ? 1 : r.plan.state_waves);
        const float* from = isA ? r.part_a : r.part_d;
        float sum = 0.0f;
        if (col < columns) {
#pragma unroll 4
            for (int k = y; k < rows; k += 16) sum += from[k * columns + col];
        }
        sums[y][x] = sum;
        __syncthreads();
        if (y == 0 && col < columns) {
            for (int i = 1; i < 16; ++i) sum += sums[i][x];
            if (isA) r.g.dA[col] = sum;
            else if (col < in.D_) { if (r.g.dD) r.g.dD[col] = sum; }
            else if (r.g.ddt_bias) r.g.ddt_bias[col - in.D_] = sum;
        }
        __syncthreads();
    }
}

struct Carve {
    size_t saved, scan, ends, steps, bc, a, d, total;
};
Carve carve(int B, int N, int D, int S, int G, bool with_saved) {
    const GradPlan p = grad_plan(B, N, D, S, G);
    const size_t rows = static_cast<size_t>(B) * p.scan.segments;
    Carve c;
    size_t off = 0;
    c.saved = off; off += with_saved ? 0 : scan_saved_bytes(B, N, D, S);
    c.scan = off; off += with_saved ? 0 : scan_workspace(B, N, D, S, G);
    c.ends = off; off += p.scan.segments > 1 ? up256(rows * quads(S) * D * 16) : 0;
    c.steps = off; off += p.scan.segments > 1 ? up256(rows * D * 4) : 0;
    c.bc = off; off += p.parts > 1 ? up256(static_cast<size_t>(p.parts) * 2 * B * N * G * S * 4) : 0;
    c.a = off; off += up256(rows * D * S * 4);
    c.d = off; off += up256(rows * p.state_waves * 2 * D * 4);
    c.total = off;
    return c;
}

template <typename T, int SP>
hipError_t back_ends(const GradRun& r, hipStream_t st) {
    const int64_t waves = static_cast<int64_t>(r.in.G) * r.plan.scan.tiles * r.in.B * r.plan.scan.segments;
    const int w = waves_together(r.in.G * r.plan.scan.tiles);
    back_ends_kernel<T, SP><<<dim3(static_cast<unsigned>(waves / w), (r.in.S + SP - 1) / SP), 64 * w, sizeof(float) * w * kP * 2 * SP, st>>>(r);
    return hipGetLastError();
}

// The kernel's LDS is asked for ahead of the call's first launch (nothing has gone out where that fails); `launch`: the kernel itself.
template <typename T, int SP, int SW>
hipError_t grad_main(const GradRun& r, bool launch, hipStream_t st) {
    const int bytes = static_cast<int>(sizeof(float)) * grad_lds<SP, SW>(r.plan.tile_waves);
    const int64_t blocks = static_cast<int64_t>(r.in.B) * r.plan.scan.segments * r.in.G * r.plan.parts;
    const auto kernel = r.in.z.data ? scan_grad_kernel<T, SP, SW, true> : scan_grad_kernel<T, SP, SW, false>;
    if (!launch) {
        static std::atomic<uint64_t> asked[2];
        if (bytes <= 65536) return hipSuccess;
        return ask_lds(reinterpret_cast<const void*>(kernel), static_cast<int>(sizeof(float)) * grad_lds<SP, SW>(SW >= 4 ? 1 : 4 / SW), asked[r.in.z.data != nullptr]);
    }
    kernel<<<static_cast<unsigned>(blocks), 64 * SW * r.plan.tile_waves, bytes, st>>>(r);
    return hipGetLastError();
}
template <typename T>
hipError_t grad_main_of(const GradRun& r, bool launch, hipStream_t st) {
    const int S = r.in.S;
    return S <= 4 ? grad_main<T, 4, 1>(r, launch, st) : S <= 8 ? grad_main<T, 8, 1>(r, launch, st) : S <= 16 ? grad_main<T, 8, 2>(r, launch, st)
           : S <= 32 ? grad_main<T, 8, 4>(r, launch, st) : grad_main<T, 8, 8>(r, launch, st);
}

// forward: the workspace of the pass that saves the states; null where they are there.
template <typename T>
hipError_t grad_of(const GradRun& r, const float* state, void* forward, hipStream_t st) {
    const int S = r.in.S;
    if (const hipError_t e = grad_main_of<T>(r, false, st); e != hipSuccess) return e;
    if (forward) {
        if (const hipError_t e = run_state_scan(std::is_same<T, float>::value ? 0 : 1, r.in, state, nullptr, nullptr, const_cast<float*>(r.saved), forward, st); e != hipSuccess) return e;
    }
    if (r.plan.scan.segments > 1) {
        if (const hipError_t e = S <= 4 ? back_ends<T, 4>(r, st) : S <= 8 ? back_ends<T, 8>(r, st) : back_ends<T, 16>(r, st); e != hipSuccess) return e;
        if (const hipError_t e = launch_join_segments(r.in, r.plan.scan, nullptr, r.ends, r.steps, true, st); e != hipSuccess) return e;
    }
    if (const hipError_t e = grad_main_of<T>(r, true, st); e != hipSuccess) return e;
    if (r.plan.parts > 1) {
        const int64_t all = static_cast<int64_t>(r.in.B) * r.in.N * r.in.G * S;
        group_sums_kernel<T><<<static_cast<unsigned>((all + 255) / 256), 256, 0, st>>>(r);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    const int a_blocks = static_cast<int>((static_cast<int64_t>(r.in.D_) * S + 63) / 64);
    const int blocks = a_blocks + (2 * r.in.D_ + 63) / 64;
    column_sums_kernel<<<blocks < kColumnBlocks ? blocks : kColumnBlocks, 1024, 0, st>>>(r, a_blocks, blocks);
    return hipGetLastError();
}

}  // namespace

size_t scan_grad_workspace(int B, int N, int D, int S, int G, bool with_saved) { return carve(B, N, D, S, G, with_saved).total; }

hipError_t launch_state_scan_grad(int dtype, AnyRows dout, const ScanIn& in, const float* state, const void* saved, const ScanGrads& g, void* ws,
                                  hipStream_t st) {
    const Carve c = carve(in.B, in.N, in.D_, in.S, in.G, saved != nullptr);
    char* base = static_cast<char*>(ws);
    const auto floats = [&](size_t off) { return reinterpret_cast<float*>(base + off); };
    if (!scan_fits(in.B, in.N, in.D_, in.S, in.G, grad_plan(in.B, in.N, in.D_, in.S, in.G).scan)) return hipErrorInvalidValue;
    const GradRun r{in, dout, g, saved ? static_cast<const float*>(saved) : floats(c.saved), floats(c.ends), floats(c.steps), floats(c.bc), floats(c.a), floats(c.d),
                    grad_plan(in.B, in.N, in.D_, in.S, in.G)};
    void* const forward = saved ? nullptr : base + c.scan;
    return dtype ? grad_of<uint16_t>(r, state, forward, st) : grad_of<float>(r, state, forward, st);
}

}  // namespace enc
}  // namespace lccrf
