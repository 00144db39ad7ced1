// Shared by the scan's forward and backward kernels: how channels, states and positions are spread, and what goes through LDS.
//
// A lane has one channel with all its states in registers; a wave 64 channels of one group, so Bm and Cm of a position are the
// same for all its lanes: a wave puts those of eight positions into LDS of its own, widened, and reads them back as
// broadcasts.  The state lives in base 2: exp(step A) = exp2(step (A log2 e)).
//
// Blocks of eight positions are worked on while the next one's inputs are on their way.  Loads and stores come back in order, and
// a wait can only leave in flight what is known to have been issued behind what it waits for.  So the next block's inputs are taken up in
// front of this block's stores, and a whole block has no condition around a store (lanes past a group's end repeat a channel
// of it and write the same value there again); only the block that ends a sequence is taken with conditions.
#pragma once

#include "lccrf_encoder.h"

#include <type_traits>

namespace lccrf {
namespace enc {

constexpr int kP = kScanBlock;

struct ScanPlan {
    int tiles;      // waves that cover a group's channels
    int all_tiles;  // and all groups' (forward pass, `flat`: tiles run on from a group into the next)
    bool flat;
    int segments;   // a sequence is cut into so many
    int seg_len;    // positions each, a multiple of kP
};

__device__ __forceinline__ int clamp_length(const int32_t* lengths, int b, int N) {
    if (!lengths) return N;
    const int n = lengths[b];
    return n < 0 ? 0 : n > N ? N : n;
}

template <typename T> __device__ __forceinline__ const T* at(const AnyRows& r, int64_t b, int64_t l) {
    return static_cast<const T*>(r.data) + b * r.batch + l * r.row;
}

// The element `bytes` behind a place that is the same for the whole wave: the address stays a scalar pair and a 32-bit offset.
template <typename T> __device__ __forceinline__ T take(const T* place, unsigned bytes) {
    return *reinterpret_cast<const T*>(reinterpret_cast<const char*>(place) + bytes);
}
template <typename T> __device__ __forceinline__ void give(T* place, unsigned bytes, float v) {
    put1(reinterpret_cast<T*>(reinterpret_cast<char*>(place) + bytes), v);
}

// A channel (its byte offset) of P rows from l0 on, `stride` apart; those past the end take the place of one before it.
template <typename T, int P> __device__ __forceinline__ void load_rows(const AnyRows& r, int b, int l0, int stride, int len, unsigned bytes, T (&v)[P]) {
    const T* p = at<T>(r, b, l0 < len ? l0 : len - 1);
#pragma unroll
    for (int i = 0; i < P; ++i) {
        v[i] = take(p, bytes);
        l0 += stride;
        p += l0 < len ? stride * r.row : 0;
    }
}
// The same where all rows lie in front of the end, p the first of them.
template <typename T, int P> __device__ __forceinline__ void load_whole(const T* p, int64_t row, unsigned bytes, T (&v)[P]) {
    asm volatile("" : "+v"(bytes));  // widened here, where the loads can use it as their offset, and not in front of the loop
#pragma unroll
    for (int i = 0; i < P; ++i, p += row) v[i] = take(p, bytes);
}

// The sequence with rank k among the lengths, the longest first (equal ones in their order).  Waves of long sequences that start
// last are what a launch waits for; where the lengths are given and a wave can look through them quickly, the
// order of work follows them.
constexpr int kMaxRanked = 256;
__device__ __forceinline__ int ranked(const int32_t* lengths, int B, int N, int k, int lane) {
    if (!lengths || B > kMaxRanked) return k;
    int len[kMaxRanked / 64], rank[kMaxRanked / 64] = {};
#pragma unroll
    for (int c = 0; c < kMaxRanked / 64; ++c) len[c] = c * 64 + lane < B ? clamp_length(lengths, c * 64 + lane, N) : -1;
    for (int j = 0; j < B; ++j) {
        const int other = clamp_length(lengths, j, N);
#pragma unroll
        for (int c = 0; c < kMaxRanked / 64; ++c) rank[c] += other > len[c] || (other == len[c] && j < c * 64 + lane);
    }
    int b = 0;
#pragma unroll
    for (int c = 0; c < kMaxRanked / 64; ++c) {
        const uint64_t hit = __ballot(rank[c] == k && c * 64 + lane < B);
        if (hit) b = c * 64 + __builtin_ctzll(hit);
    }
    return b;
}

// Waves have nothing to do with each other; workgroups of four are what they come in where the tiles are a multiple of four (saving
// forward pass of B=128 N=256 D=1024 S=16, ragged: 132 us, 152 in workgroups of one), else of one, so that every wave has a tile
// and the SIMDs fill evenly (B=4 N=16384 D=514 in two groups, ten tiles: 286 us, 386 in workgroups of four).
inline int waves_together(int tiles) { return tiles % 4 == 0 ? 4 : 1; }

__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// exp2's argument of a state: A log2(e), kept finite so that a step of 0 (positions past the end) leaves the state as it is.
__device__ __forceinline__ float base2(float A) {
    const float a = A * kLog2e;
    return a < -3.0e38f ? -3.0e38f : a;
}

// Kernels hold 4 quads(S) states a channel.  Places past S hold states of the front once more (one state: four times), each of the
// copies, as many as a power of two, with its share of Cm: what they add up to is exact, by way of the gradients too, and infinite or NaN where the
// states by themselves are.  Places of zeros would make NaN of an infinite x, step or gradient.
__host__ __device__ inline int quads(int S) { return S <= 4 ? 1 : S <= 8 ? 2 : S <= 16 ? 4 : S <= 32 ? 8 : 16; }
__device__ __forceinline__ int state_at(int place, int S) { return place < S ? place : S == 1 ? 0 : place - S; }
__device__ __forceinline__ float copies_of(int s, int S) { return S == 1 ? 4.0f : s + S < 4 * quads(S) ? 2.0f : 1.0f; }

// Bm and Cm of kP positions for the states s0 .. s0 + SP - 1, on their way from memory to LDS [kP][2 * SP] (Bm, then Cm).
// Positions past the end count as 0.  A lane has state lane % SP of the positions lane / SP + i * kStep.
template <typename T, int SP> struct GroupVectors {
    static constexpr int R = kP * SP / 64 ? kP * SP / 64 : 1, kStep = 64 / SP;
    T vb[R], vc[R];
    const T *pb, *pc;  // of this lane's first position
    int first;
    float share;  // of its state's copies, for Cm
    __device__ __forceinline__ void place(const ScanIn& in, int b, int l0, int group, int s0, int lane) {
        const int s = state_at(s0 + lane % SP, in.S);
        first = lane / SP % kP;
        share = 1.0f / copies_of(s, in.S);
        pb = at<T>(in.Bm, b, l0 + first) + group * in.b_group + s;
        pc = at<T>(in.Cm, b, l0 + first) + group * in.c_group + s;
    }
    // A block that the end may lie in: past it the last position stands in.
    __device__ __forceinline__ void load(const ScanIn& in, int l0, int len) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int l = l0 + first + i * kStep, back = l < len ? 0 : l - (len - 1);
            vb[i] = pb[(i * kStep - back) * in.Bm.row];
            vc[i] = pc[(i * kStep - back) * in.Cm.row];
        }
    }
    // The whole block that lies `blocks` further.
    __device__ __forceinline__ void next(const ScanIn& in, int blocks) {
        pb += blocks * kP * in.Bm.row;
        pc += blocks * kP * in.Cm.row;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            vb[i] = pb[i * kStep * in.Bm.row];
            vc[i] = pc[i * kStep * in.Cm.row];
        }
    }
    template <bool WHOLE> __device__ __forceinline__ void put(float* lds, int l0, int len, int lane) const {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int pos = first + i * kStep;
            const bool is = WHOLE || l0 + pos < len;
            lds[pos * 2 * SP + lane % SP] = is ? widen(vb[i]) : 0.0f;
            lds[pos * 2 * SP + SP + lane % SP] = is ? widen(vc[i]) * share : 0.0f;
        }
    }
};

// Saved states: [B][ceil(N / kP)][quads][D][4] floats, the states rounded up to what a kernel holds.
__device__ __forceinline__ int64_t quad_at(int64_t block, int S, int D, int q, int d) { return ((block * quads(S) + q) * D + d) * 4; }

// The same as a place for the whole wave and a byte offset (a channel's 16 bytes; D <= 2^22).
__device__ __forceinline__ unsigned quad_bytes(int D, int q, int d) { return (static_cast<unsigned>(q) * D + d) * 16; }

// Where the segment that starts at `begin` ends (the last one's full length may reach past 32 bits).
__device__ __forceinline__ int segment_stop(const ScanPlan& p, int begin, int N) { return N - begin < p.seg_len ? N : begin + p.seg_len; }

inline int scan_blocks(int N) { return (N + kP - 1) / kP; }

// Segments: the recursion over a segment needs the state in front of it, which takes a pass of its own over all segments (eight
// tenths of the forward work again, two of the gradient's) and a short one along them.  That pays where the waves that the batch has by
// itself leave most of the chip empty: a lone wave issues an instruction where two issue three, so one segment costs 1.5 a position where
// the segments of 2048 waves (two a SIMD, `room`; never a few more than that, which would take a third as long again) cost 1.8 over their number.
// B=4 N=16384 D=514 S=16, 36 waves by itself: 56 segments 259 us, one 4399.
inline ScanPlan scan_plan(int B, int N, int D, int G, bool flat, int waves_a_tile, int room, int least) {
    ScanPlan p;
    p.tiles = (D / G + 63) / 64;
    p.flat = flat;
    p.all_tiles = flat ? (D + 63) / 64 : G * p.tiles;
    const int64_t waves = static_cast<int64_t>(B) * p.all_tiles * waves_a_tile;
    int64_t segments = room / waves;
    if (segments < least) segments = 1;
    const int64_t most = (N + 63) / 64;
    if (segments > most) segments = most;
    p.seg_len = static_cast<int>(((N + segments - 1) / segments + kP - 1) / kP * kP);
    p.segments = static_cast<int>((static_cast<int64_t>(N) + p.seg_len - 1) / p.seg_len);
    return p;
}
// Groups of 64 channels and more whose tiles would not be full (up to 16 states): tiles run on into the next group, and a wave holds the
// vectors of two (B=4 N=16384, two groups of 257 channels, nine tiles instead of ten: 282 -> 265 us).
inline ScanPlan forward_plan(int B, int N, int D, int S, int G) {
    const bool flat = S <= 16 && D / G >= 64 && (D + 63) / 64 < G * ((D / G + 63) / 64);
    return scan_plan(B, N, D, G, flat, S <= 16 ? 1 : S <= 32 ? 2 : 4, 2048, 3);
}

inline bool scan_fits(int B, int N, int D, int S, int G, const ScanPlan& p) {
    const int64_t most = (int64_t{1} << 32) - 1024, b = B;
    return b * p.segments * p.all_tiles * 512 < most && b * D * quads(S) < most && b * N * G * S < most;
}

// Runs the scan for the saved states alone (out and final_state null), or with them.
hipError_t run_state_scan(int dtype, const ScanIn& in, const float* state, void* out, float* final_state, float* saved, void* ws, hipStream_t st);
// The pass along the segments: ends [B][segments][quads][D][4] of every segment from 0 become what stands at its beginning
// (back: at its end).  state: [B][D][S] in front of the first, or null.
hipError_t launch_join_segments(const ScanIn& in, const ScanPlan& p, const float* state, float* ends, const float* steps, bool back, hipStream_t st);

}  // namespace enc
}  // namespace lccrf
