// Shared by the gated recurrence's forward and backward kernels: how channels and positions are spread, and the gates.
//
// h = a h + b is a recursion in one number a channel: little arithmetic, so the traffic is what has to bound it, and for that
// positions have to be worked on side by side.  A workgroup has a tile of 64 V channels and goes through a sequence in blocks of W P
// positions: each of its W waves takes P of them, makes (A, E) of them - what they turn a state h into, A h + E - and puts that into LDS;
// after one barrier every wave folds the waves' pairs in front of it onto the state before the block and runs its own positions again from there, with
// the a and b that it has kept in registers.  So every input is read once and its gates are computed once.
#pragma once

#include "lccrf_layers.h"

namespace lccrf {
namespace enc {

constexpr int kRecurSave = 32;   // positions between two saved states
constexpr int kRecurBlock = 64;  // segments are multiples of it

struct RecurPlan {
    int tiles, segments, seg_len;
};

// V channels of a row.
template <typename T, int V> using Bit = Piece<T, V, V == 1>;

template <typename T> __device__ __forceinline__ const T* row_of(const AnyRows& r, int64_t b, int64_t l) {
    return static_cast<const T*>(r.data) + b * r.batch + l * r.row;
}

// Which channels a lane has.  The last lane of an odd width starts one channel early, at one that the lane before has too, and
// gives nothing of it away (the state may be written in place: what it computes there need not be right).
template <int V> struct Lane {
    int c;              // first channel
    bool all, last;     // gives all V of them, the last one alone
    bool full;          // (the same for the whole tile) every lane gives all
    __device__ __forceinline__ Lane(int tile, int lane, int D) {
        const int want = (tile * 64 + lane) * V;
        c = want <= D - V ? want : D - V;
        all = want <= D - V;
        last = V > 1 && !all && want < D;
        full = (tile + 1) * 64 * V <= D;
    }
    template <typename T> __device__ __forceinline__ void give(T* row, const float (&v)[V]) const {
        T* p = reinterpret_cast<T*>(reinterpret_cast<char*>(row) + static_cast<unsigned>(c) * sizeof(T));
        if (full || all) Bit<T, V>::put(p, V, v);
        else if (last) put1(p + V - 1, v[V - 1]);
    }
};

template <typename T, int V> __device__ __forceinline__ void take_bit(Bit<T, V>& v, const T* row, unsigned bytes) {
    v.load(reinterpret_cast<const T*>(reinterpret_cast<const char*>(row) + bytes), V);
}

// P rows from l0 on; those at or past the end take the place of the last one before it (len > 0).
template <typename T, int V, int P> __device__ __forceinline__ void take_rows(Bit<T, V> (&v)[P], const AnyRows& r, int b, int l0, int len, unsigned bytes) {
    const T* p = row_of<T>(r, b, l0 < len ? l0 : len - 1);
#pragma unroll
    for (int i = 0; i < P; ++i) {
        take_bit<T, V>(v[i], p, bytes);
        p += l0 + i + 1 < len ? r.row : 0;
    }
}

struct RecurChannel { float c, f_bias, g_bias; };  // c = -rate log(1 + exp(decay))
__device__ __forceinline__ RecurChannel recur_channel(const RecurIn& in, int d) {
    return {-in.rate * softplus(in.decay[d]).value, in.f_bias ? in.f_bias[d] : 0.0f, in.g_bias ? in.g_bias[d] : 0.0f};
}

// u = c open and a = exp(u); rest = 1 - a^2.  For small u, a^2 has lost what 1 - a^2 is made of: from 2 u > -1/4 on the series of
// 1 - exp(2 u) instead (off by less than 2^-25 of it), below that 1 - a a loses no more than two bits.
struct Decay { float open, a, rest; };
__device__ __forceinline__ Decay decay_of(float f, const RecurChannel& ch) {
    Decay d;
    d.open = sigmoid(f + ch.f_bias);
    const float u = ch.c * d.open, v = 2.0f * u;
    d.a = exp2_fast(u * kLog2e);
    float q = 1.0f / 720.0f;
    q = fmaf(q, v, 1.0f / 120.0f);
    q = fmaf(q, v, 1.0f / 24.0f);
    q = fmaf(q, v, 1.0f / 6.0f);
    q = fmaf(q, v, 0.5f);
    q = fmaf(q, v, 1.0f);
    d.rest = v > -0.25f ? -v * q : fmaf(-d.a, d.a, 1.0f);
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

inline size_t recur_ends_bytes(int B, int segments, int D) { return up256(static_cast<size_t>(B) * segments * D * 8); }

}  // namespace enc
}  // namespace lccrf
