// Shared by the encoder's kernels (embedding, short convolution, state space scan): element types, vectors that
// need no more than an element's alignment, the functions of the gates, argument blocks and launch entry points.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>

namespace lccrf {
namespace enc {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2f = 0.69314718055994530942f;

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Rounded once, to nearest even (one instruction on gfx950).
__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x)); }
__device__ __forceinline__ uint32_t to_bf16_pair(float low, float high) {  // both by one instruction
    typedef float Floats __attribute__((ext_vector_type(2)));
    typedef __bf16 Halves __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(Floats{low, high}, Halves));
}
__device__ __forceinline__ float from_bf16(uint16_t h) { return __uint_as_float(static_cast<uint32_t>(h) << 16); }

__device__ __forceinline__ float get1(const float* p) { return *p; }
__device__ __forceinline__ float get1(const uint16_t* p) { return from_bf16(*p); }
__device__ __forceinline__ void put1(float* p, float v) { *p = v; }
__device__ __forceinline__ void put1(uint16_t* p, float v) { *p = to_bf16(v); }
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(uint16_t v) { return from_bf16(v); }

// Elements of a 16-byte vector.
template <typename T> struct Wide { static constexpr int V = 16 / sizeof(T); };

// A piece of a row: W consecutive channels at an address aligned like one element (the hardware takes such wide accesses as they
// are), loaded first and widened where it is used, so that loads stay in flight.  Rows whose width is no multiple of W
// have their last piece moved back to end with the row (piece_start): it and the one before share some channels, and
// compute and write the same values there.  SMALL: rows narrower than a piece, element by element.
template <int WORDS> struct Words { typedef uint32_t v __attribute__((ext_vector_type(WORDS))); };
template <typename T, int W, bool SMALL = false> struct Piece {
    typedef typename Words<W * sizeof(T) / 4>::v Vec;
    typedef Vec Any __attribute__((aligned(sizeof(T))));
    Vec raw;
    __device__ __forceinline__ void load(const T* p, int) { raw = *reinterpret_cast<const Any*>(p); }
    __device__ __forceinline__ void get(float (&o)[W]) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < W; ++i) o[i] = __uint_as_float(raw[i]);
        } else {
#pragma unroll
            for (int i = 0; i < W / 2; ++i) {
                o[2 * i] = __uint_as_float(raw[i] << 16);
                o[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
            }
        }
    }
    template <bool STREAM = false> static __device__ __forceinline__ void put(T* p, int, const float (&o)[W]) {
        Vec v;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] = __float_as_uint(o[i]);
        } else {
#pragma unroll
            for (int i = 0; i < W / 2; ++i) v[i] = to_bf16_pair(o[2 * i], o[2 * i + 1]);
        }
        if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<Any*>(p));
        else *reinterpret_cast<Any*>(p) = v;
    }
};
template <typename T, int W> struct Piece<T, W, true> {
    T raw[W];
    __device__ __forceinline__ void load(const T* p, int D) {
#pragma unroll
        for (int i = 0; i < W; ++i) raw[i] = i < D ? p[i] : T(0);
    }
    __device__ __forceinline__ void get(float (&o)[W]) const {
#pragma unroll
        for (int i = 0; i < W; ++i) o[i] = widen(raw[i]);
    }
    template <bool STREAM = false> static __device__ __forceinline__ void put(T* p, int D, const float (&o)[W]) {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < D) put1(p + i, o[i]);
    }
};
template <int W, bool SMALL> __device__ __forceinline__ int piece_start(int piece, int D) {
    if (SMALL) return 0;
    return piece * W <= D - W ? piece * W : D - W;
}
// Pieces of a row (D up to 2^31 - 1: nothing here or above goes past it).
__host__ __device__ inline int pieces_of_row(int D, int W) { return (D - 1) / W + 1; }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + exp2_fast(-x * kLog2e)); }
// The gate by itself, to be multiplied in afterwards: |silu| <= |x|, where a value times x could pass the largest float on its way to a number.
__device__ __forceinline__ float silu(float x) { return x * sigmoid(x); }

// log(1 + exp(v)) and its derivative.  With e = exp(-|v|): max(v, 0) + log1p(e), and log1p(e) = e (1 + e q(e)) with q of degree 8
// fitted to it on [0, 1] (off by at most 1.4 units in the last place): a logarithm of 1 + e would lose the steps near 0.001 that
// such scans live on.  e is exp2(t), t = -|v| log2(e) rounded, times 1 + (-|v| - t ln2): the rounding of t alone would cost 2^-20
// at |v| = 16.  exp(-126) is 0 in float already, so -|v| may stop there; a NaN stays one
// (this maximum, unlike fmaxf, hands it on).
struct Softplus { float value, slope; };
__device__ __forceinline__ Softplus softplus(float v) {
    const float a = fmaxf(-fabsf(v), -126.0f);
    const float t = a * kLog2e;
    const float rest = fmaf(t, 1.9046542999577680e-9f, fmaf(t, -0.693147182464599609375f, a));  // ln2 in two parts
    float e = exp2_fast(t);
    e = fmaf(e, rest, e);
    float q = -0.004579766187816858f;
    q = fmaf(q, e, 0.025682786479592323f);
    q = fmaf(q, e, -0.06751181185245514f);
    q = fmaf(q, e, 0.11626528203487396f);
    q = fmaf(q, e, -0.15878385305404663f);
    q = fmaf(q, e, 0.19862109422683716f);
    q = fmaf(q, e, -0.2498755156993866f);
    q = fmaf(q, e, 0.3333289325237274f);
    q = fmaf(q, e, -0.49999997f);
    q = fmaf(q, e, 1.0f);
    const float r = __builtin_amdgcn_rcpf(1.0f + e);
    return {fmaf(q, e, __builtin_elementwise_maximum(v, 0.0f)), v >= 0.0f ? r : e * r};
}

// Rows of an input: element strides between sequences and positions.
template <typename T> struct Rows {
    const T* data;
    int64_t batch, row;
};
struct AnyRows {
    const void* data;
    int64_t batch, row;
    template <typename T> __host__ __device__ Rows<T> as() const { return {static_cast<const T*>(data), batch, row}; }
};

// The argument block of the scan's kernels.
struct ScanIn {
    AnyRows x, dt, Bm, Cm, z;
    int64_t b_group, c_group;
    const float *A, *D, *dt_bias;
    const int32_t* lengths;
    int B, N, D_, S, G;
};
struct ScanGrads {
    void *dx, *ddt, *dBm, *dCm, *dz;
    float *dA, *dD, *ddt_bias, *dstate;
};

// Of a call of the convolution or scan.  Kernels count positions in 32 bits, and go past a sequence's end by less than a run or a block.
constexpr int64_t kMaxPositions = (int64_t{1} << 31) - 1024;

constexpr int kScanBlock = 8;  // positions between two saved states

// dtype 0: float, 1: bfloat16.  All return the status of their launches.
hipError_t launch_embed(int dtype, const void* table, int V, int D, int64_t table_row, const int32_t* ids, int64_t n, float scale, void* out, hipStream_t st);
size_t embed_grad_workspace(int64_t n, int V, int D);
hipError_t launch_embed_grad(int dtype, AnyRows dout, const int32_t* ids, int B, int N, int V, int D, float scale, void* grad, void* ws, hipStream_t st);

hipError_t launch_conv(int dtype, AnyRows x, const float* weight, const float* bias, const void* state, const int32_t* lengths, int B, int N, int D, int K,
                       void* out, void* final_state, hipStream_t st);
size_t conv_grad_workspace(int B, int N, int D, int K);
hipError_t launch_conv_grad(int dtype, AnyRows dout, AnyRows x, const float* weight, const float* bias, const void* state, const int32_t* lengths, int B, int N,
                            int D, int K, void* dx, float* dweight, float* dbias, void* dstate, void* ws, hipStream_t st);
hipError_t launch_conv_step(int dtype, const void* x, int64_t x_row, const float* weight, const float* bias, void* state, int B, int D, int K, void* out,
                            hipStream_t st);

size_t scan_saved_bytes(int B, int N, int D, int S);
size_t scan_workspace(int B, int N, int D, int S, int G);
size_t scan_grad_workspace(int B, int N, int D, int S, int G, bool with_saved);
hipError_t launch_state_scan(int dtype, const ScanIn& in, const float* state, void* out, float* final_state, void* saved, void* ws, hipStream_t st);
hipError_t launch_state_scan_grad(int dtype, AnyRows dout, const ScanIn& in, const float* state, const void* saved, const ScanGrads& g, void* ws,
                                  hipStream_t st);
hipError_t launch_state_step(int dtype, const ScanIn& in, float* state, void* out, hipStream_t st);

// Results that the L2 caches could not hold (eight of 4 MB) are written past them, us past / through them (inputs and results in turn in
// several places): lookup of 67 MB 13.7 / 23.1; embedding gradient of 205 MB 76 / 96; convolutions of 67 MB 35 / 41, 134 MB 62.5 / 64.4, 268 MB
// 106 / 110, 537 MB 232 / 235, of 66 MB with an odd width 41 / 47; convolution and gradient of 134 MB each 147 / 157.
inline bool past_caches(int64_t bytes) { return bytes > (int64_t{32} << 20); }
// A launch has fewer than 2^32 threads; the entry points refuse what would take more, before anything is enqueued.  The sums over
// columns behind a gradient would pass that where nothing else does: at most kColumnBlocks workgroups take their blocks of columns in turn.
constexpr int kColumnBlocks = 1 << 16;
inline bool fits(int64_t blocks, int threads) { return blocks * threads < (int64_t{1} << 32); }
// More than 64 KB of LDS has to be asked for, once a kernel and device (`asked`: a bit a device).
inline hipError_t ask_lds(const void* kernel, int bytes, std::atomic<uint64_t>& asked) {
    int dev = 0;
    if (const hipError_t e = hipGetDevice(&dev); e != hipSuccess) return e;
    const uint64_t bit = uint64_t{1} << (dev & 63);
    if (asked.load(std::memory_order_relaxed) & bit) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) asked.fetch_or(bit, std::memory_order_relaxed);
    return e;
}
inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace enc
}  // namespace lccrf
