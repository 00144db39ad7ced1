// Shared by the gated recurrence's forward and backward kernels: how channels and positions are spread, and the gates.
//
// h = a h + b is a recursion in one number a channel: little arithmetic, so the traffic is what has to bound it, and for that
// positions have to be worked on side by side.  A workgroup has a tile of channels and goes through a sequence in blocks of positions: a wave
// has 64 / SUB lanes across the tile, V channels each, and SUB sets of them, every one with P positions of the block.  A lane makes (A, E)
// of its positions - what they turn a state h into, A h + E; those of a wave are joined by shuffles, those of the waves through LDS: after one barrier every
// wave folds the pairs of the waves in front of it onto the state before the block, and every lane runs its own positions again from there, with the
// a and b that it has kept in registers; the last one leaves the state behind the block in LDS.  So every input is read once and its gates
// are computed once.  Narrow tiles (SUB 4) are for few sequences, where wide ones would be fewer workgroups than the chip has room for.
#pragma once

#include "lccrf_layers.h"

namespace lccrf {
namespace enc {

constexpr int kRecurSave = 8;   // positions between two saved states
constexpr int kRecurBlock = 64;  // segments are multiples of it

constexpr int kWideTile = 128, kNarrowTile = 32;  // channels
struct RecurPlan {
    bool narrow;
    int tiles, segments, seg_len;
    bool near;  // tiles of the same positions on one XCD
};

// Workgroups with neighbouring blockIdx run on different ones of the eight XCDs, each with an L2 of its own.  Tiles of the same positions lie next to each
// other and share the cache lines on their borders (where a row is no whole number of lines, most of them): eight sequences' segments side by side, all tiles
// of each on one XCD.
constexpr int kXcds = 8;
struct RecurWork { int b, seg, tile; };  // (in scalar registers, though divided for in vector ones)
__device__ __forceinline__ RecurWork recur_work(const RecurPlan& p) {
    const unsigned tiles = p.tiles, segments = p.segments, rest = p.near ? blockIdx.x / kXcds : blockIdx.x, group = rest / tiles;
    const unsigned which = p.near ? group * kXcds + blockIdx.x % kXcds : group, b = which / segments;
    return {__builtin_amdgcn_readfirstlane(static_cast<int>(b)), __builtin_amdgcn_readfirstlane(static_cast<int>(which - b * segments)),
            __builtin_amdgcn_readfirstlane(static_cast<int>(rest - group * tiles))};
}
inline int64_t recur_blocks(const RecurPlan& p, int B) {
    const int64_t all = static_cast<int64_t>(B) * p.segments;
    return (p.near ? (all + kXcds - 1) / kXcds * kXcds : all) * p.tiles;
}

// Wide tiles (`many` workgroups of them fill the chip), else narrow ones for sequences that are not long, else wide tiles of segments: a pass of its own
// over all segments makes what each turns a state into, and the segments side by side fold those in front of them.  (How many of which: with the launches.)
inline RecurPlan recur_plan_of(int B, int N, int D, int many, int narrow, int longest) {
    RecurPlan p;
    p.narrow = false;
    p.tiles = (D - 1) / (D == 1 ? 64 : kWideTile) + 1;
    const int64_t groups = static_cast<int64_t>(B) * p.tiles;
    int64_t segments = 1;
    if (groups < many) {
        const int64_t tiles = (D - 1) / kNarrowTile + 1;
        if (D > 1 && (N <= longest || B * tiles >= narrow)) {
            p.narrow = true;
            p.tiles = static_cast<int>(tiles);
        } else {
            segments = 2048 / groups;
        }
    }
    const int64_t most = (static_cast<int64_t>(N) + kRecurBlock - 1) / kRecurBlock;
    if (segments > most) segments = most;
    if (segments < 1) segments = 1;
    p.seg_len = static_cast<int>(((N + segments - 1) / segments + kRecurBlock - 1) / kRecurBlock * kRecurBlock);
    p.segments = static_cast<int>((static_cast<int64_t>(N) + p.seg_len - 1) / p.seg_len);
    p.near = static_cast<int64_t>(B) * p.segments >= 8 * kXcds;
    return p;
}

// V channels of a row.
template <typename T, int V> using Bit = Piece<T, V, V == 1>;

template <typename T> __device__ __forceinline__ const T* row_of(const AnyRows& r, int64_t b, int64_t l) {
    return static_cast<const T*>(r.data) + b * r.batch + l * r.row;
}

// Which channels a lane has.  Where the width is no multiple of V the last lane's are moved back to end with the row: those that the lane
// before has too it gives nothing away of (the state may be written in place: what it computes there need not be right).
template <int V> struct Lane {
    int c, own;  // first channel; how many, from the last one on, are its own
    bool full;   // (the same for the whole tile) every lane has V of its own
    __device__ __forceinline__ Lane(int tile, int lane, int lanes, int D) {
        const int want = (tile * lanes + lane) * V, left = D - want;
        c = left >= V ? want : D - V;
        own = left >= V ? V : left > 0 ? left : 0;
        full = (tile + 1) * lanes * V <= D;
    }
    // (`at`: this lane's row, so many elements behind the wave's.)  The offset is added by the store itself, not to every output's address ahead of a loop.
    template <bool WHOLE = false, typename T> __device__ __forceinline__ void give(T* row, const float (&v)[V], unsigned at = 0) const {
        unsigned bytes = (at + static_cast<unsigned>(c)) * static_cast<unsigned>(sizeof(T));
        asm volatile("" : "+v"(bytes));
        T* p = reinterpret_cast<T*>(reinterpret_cast<char*>(row) + bytes);
        if (WHOLE || own == V) {
            Bit<T, V>::put(p, V, v);
        } else {
#pragma unroll
            for (int j = 1; j < V; ++j)
                if (j >= V - own) put1(p + j, v[j]);
        }
    }
};

template <typename T, int V> __device__ __forceinline__ void take_bit(Bit<T, V>& v, const T* row, unsigned bytes) {
    v.load(reinterpret_cast<const T*>(reinterpret_cast<const char*>(row) + bytes), V);
}

// P rows, from `first` on for the wave's first set of lanes and P further for each of the next; of those at or past the end the last one before it
// (len > 0) takes the place.  A lane's place is a scalar address and a 32-bit offset: `set` is P times its number of set, `step` the bytes from a row to
// the next (near_rows below), `bytes` its channels'.
template <typename T, int V, int P, int SUB, bool WHOLE = false>
__device__ __forceinline__ void take_rows(Bit<T, V> (&v)[P], const AnyRows& r, int b, int first, int len, int set, unsigned bytes) {
    const unsigned step = static_cast<unsigned>(r.row) * sizeof(T);
    if (WHOLE || first + P * SUB <= len) {
        const T* p = row_of<T>(r, b, first);
        const unsigned at = SUB > 1 ? set * step + bytes : bytes;
#pragma unroll
        for (int i = 0; i < P; ++i, p += r.row) take_bit<T, V>(v[i], p, at);
    } else {
        const int most = first < len ? len - 1 - first : 0;
        const T* p = row_of<T>(r, b, first < len ? first : len - 1);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (SUB > 1) take_bit<T, V>(v[i], p, static_cast<unsigned>(set + i < most ? set + i : most) * step + bytes);
            else take_bit<T, V>(v[i], p + (i < most ? i : most) * r.row, bytes);
        }
    }
}
// Rows of a wave no further apart than its 32-bit offsets reach; with others, tiles are wide.
inline bool near_rows(const AnyRows& r) { return r.row >= 0 && r.row < (1 << 24); }
inline void widen_tiles(RecurPlan& p, int D) {
    if (p.narrow) p.tiles = (D - 1) / kWideTile + 1;
    p.narrow = false;
}

// A channel's constants, times log2(e) where they go into a power of two: c = -rate log(1 + exp(decay)).
struct RecurChannel { float c, f_bias, g_bias; };
__device__ __forceinline__ RecurChannel recur_channel(const RecurIn& in, int d) {
    return {-in.rate * softplus(in.decay[d]).value * kLog2e, in.f_bias ? -kLog2e * in.f_bias[d] : 0.0f, in.g_bias ? -kLog2e * in.g_bias[d] : 0.0f};
}
// s(v + bias), bias times -log2(e).
__device__ __forceinline__ float open_gate(float v, float bias) { return __builtin_amdgcn_rcpf(1.0f + exp2_fast(fmaf(v, -kLog2e, bias))); }

// a = exp(u) = exp2(t), t = c open; rest = 1 - a^2.  For small u, a^2 has lost what 1 - a^2 is made of: from 2 u > -1/4 on
// a polynomial instead, t q(t), q of degree 4 through (1 - exp(2 u)) / t at Chebyshev's points (with its rounded coefficients off by at most 2^-26 of it); below that
// 1 - a a loses no more than two bits.
struct Decay { float open, t, a, rest; };
__device__ __forceinline__ Decay decay_of(float f, const RecurChannel& ch) {
    Decay d;
    d.open = open_gate(f, ch.f_bias);
    d.t = ch.c * d.open;
    d.a = exp2_fast(d.t);
    float q = -0.0384703129529953f;
    q = fmaf(q, d.t, -0.15323998034000397f);
    q = fmaf(q, d.t, -0.44399136304855347f);
    q = fmaf(q, d.t, -0.9609050750732422f);
    q = fmaf(q, d.t, -1.3862943649291992f);
    d.rest = d.t > -0.18033688f ? q * d.t : fmaf(-d.a, d.a, 1.0f);
    return d;
}

// A product of decays: where it falls below every float though no factor is 0, it stays the least one above 0, so that an infinite state stays
// infinite over many positions as it does over each of them.
__device__ __forceinline__ float product(float p, float q) {
    const float r = p * q;
    return r == 0.0f && p != 0.0f && q != 0.0f ? 1.401298464e-45f : r;
}
template <int P, int V> __device__ __forceinline__ float product_of(const float (&a)[P][V], int j) {
    float r = a[0][j];
#pragma unroll
    for (int i = 1; i < P; ++i) r *= a[i][j];
    if (r == 0.0f) {
        bool zero = false;
#pragma unroll
        for (int i = 0; i < P; ++i) zero = zero || a[i][j] == 0.0f;
        r = zero ? 0.0f : 1.401298464e-45f;
    }
    return r;
}

// Pairs (A, E) of a wave's SUB sets of lanes: what the sets in front of a lane's own make of a state (BACK: behind it, on the way back).
template <int SUB, bool BACK> __device__ __forceinline__ void before_set(float& A, float& E, int set) {
    constexpr int L = 64 / SUB;
    if (SUB == 1) {
        A = 1.0f;
        E = 0.0f;
        return;
    }
    const int rank = BACK ? SUB - 1 - set : set;
#pragma unroll
    for (int d = 1; d < SUB; d *= 2) {
        const float a = BACK ? __shfl_down(A, d * L) : __shfl_up(A, d * L), e = BACK ? __shfl_down(E, d * L) : __shfl_up(E, d * L);
        if (rank >= d) {
            E = fmaf(A, e, E);
            A = product(A, a);
        }
    }
    const float a = BACK ? __shfl_down(A, L) : __shfl_up(A, L), e = BACK ? __shfl_down(E, L) : __shfl_up(E, L);
    A = rank ? a : 1.0f;
    E = rank ? e : 0.0f;
}

inline size_t recur_ends_bytes(int B, int segments, int D) { return up256(static_cast<size_t>(B) * segments * D * 8); }

}  // namespace enc
}  // namespace lccrf
