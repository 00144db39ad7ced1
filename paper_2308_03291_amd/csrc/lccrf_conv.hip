// Short causal convolution, its gradient and its single-token form.
//
// K products an output: the traffic of the input read and the output written once is what bounds all three.  A thread has a
// 16-byte piece of the channels and walks along a run of positions, its K last inputs in registers, so an input is read
// once but for the K - 1 in front of every run (which another thread has just read).  Measured, inputs cold: forward B=64 N=512 D=2048
// bfloat16, 270 MB, 61.5 us (4.4 TB/s); forward and gradient of B=128 N=128 D=1001 float, ragged, 207 MB, 74.5 us (padding goes through the gradient's
// arithmetic like any position).  A step of 64 streams with D=2048 takes the kernel 3.4 us, its launch and the call more.
#include "lccrf_encoder.h"

namespace lccrf {
namespace enc {
namespace {

struct ConvArgs {
    AnyRows x, dout;
    const float *weight, *bias;
    const void* state;
    const int32_t* lengths;
    int B, N, D, cpr, run, runs;  // cpr pieces a row; `runs` runs of `run` positions a sequence
};

__device__ __forceinline__ int length_of(const int32_t* lengths, int b, int N) {
    if (!lengths) return N;
    const int n = lengths[b];
    return n < 0 ? 0 : n > N ? N : n;
}

// Input l of sequence b (l >= 1 - K; below 0: of the state).  What is not there (past the end, no state) is loaded from a
// place that is and then not taken: no branch stands between the loads.
template <typename T, int K, int W, bool SMALL>
struct Input {
    Piece<T, W, SMALL> piece;
    bool is;
    __device__ __forceinline__ void load(const ConvArgs& a, int b, int l, int len, int c) {
        const T* state = static_cast<const T*>(a.state);
        is = l >= 0 ? l < len : state != nullptr;
        const T* p = l >= 0 ? static_cast<const T*>(a.x.data) + b * a.x.batch + l * a.x.row + c
                            : state + (static_cast<int64_t>(b) * (K - 1) + (l + K - 1)) * a.D + c;
        piece.load(is ? p : reinterpret_cast<const T*>(a.weight), a.D);
    }
    __device__ __forceinline__ void get(float (&v)[W]) const {
        piece.get(v);
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] = is ? v[j] : 0.0f;
    }
};

template <int K, int W>
__device__ __forceinline__ void taps_of(const ConvArgs& a, int c, float (&w)[K][W], float (&bias)[W]) {
#pragma unroll
    for (int j = 0; j < W; ++j) {
        const bool is = c + j < a.D;
        bias[j] = is && a.bias ? a.bias[c + j] : 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) w[k][j] = is ? a.weight[static_cast<int64_t>(c + j) * K + k] : 0.0f;
    }
}

template <int K> struct Group { static constexpr int U = K >= 4 ? K : K == 3 ? 6 : 4; };  // positions in flight: a multiple of K

template <typename T, int K, bool SMALL, bool STREAM>
__global__ __launch_bounds__(256) void conv_kernel(ConvArgs a, T* __restrict__ out, T* __restrict__ final_state) {
    constexpr int W = Wide<T>::V, U = Group<K>::U;
    using P = Piece<T, W, SMALL>;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t row = id / a.cpr;
    if (row >= static_cast<int64_t>(a.B) * a.runs) return;
    const int c = piece_start<W, SMALL>(static_cast<int>(id - row * a.cpr), a.D);
    const int b = static_cast<int>(row / a.runs), r = static_cast<int>(row - static_cast<int64_t>(b) * a.runs);
    const int len = length_of(a.lengths, b, a.N), l0 = r * a.run, l1 = l0 + a.run < a.N ? l0 + a.run : a.N;
    T* o = out + (static_cast<int64_t>(b) * a.N) * a.D + c;
    if (l0 < len) {
        float w[K][W], bias[W], ring[K][W];  // ring[l mod K]: input l (l0 is a multiple of U, so of K)
        Input<T, K, W, SMALL> v[U];
        taps_of<K, W>(a, c, w, bias);
#pragma unroll
        for (int k = 1; k < K; ++k) v[k - 1].load(a, b, l0 - K + k, len, c);
#pragma unroll
        for (int k = 1; k < K; ++k) v[k - 1].get(ring[k]);
        for (int l = l0; l < l1; l += U) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u].load(a, b, l + u, len, c);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float res[W];
                v[u].get(ring[u % K]);
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    float pre = bias[j];
#pragma unroll
                    for (int k = 0; k < K; ++k) pre = fmaf(w[k][j], ring[(u + 1 + k) % K][j], pre);
                    res[j] = l + u < len ? pre * sigmoid(pre) : 0.0f;
                }
                if (l + u < l1) P::template put<STREAM>(o + static_cast<int64_t>(l + u) * a.D, a.D, res);
            }
        }
    } else {
        const float zero[W] = {};
        for (int l = l0; l < l1; ++l) P::template put<STREAM>(o + static_cast<int64_t>(l) * a.D, a.D, zero);
    }
    if (r == 0 && final_state) {
#pragma unroll
        for (int k = 0; k < K - 1; ++k) {
            float v[W];
            Input<T, K, W, SMALL> in;
            in.load(a, b, len - (K - 1) + k, len, c);
            in.get(v);
            P::put(final_state + (static_cast<int64_t>(b) * (K - 1) + k) * a.D + c, a.D, v);
        }
    }
}

// Gradient.  A thread passes over a run of positions and the K - 1 behind it: dpre[l] of the whole window gives dx, those of
// its own run the sums for weight and bias.  Workgroups are lx pieces wide and 256 / lx runs high; the sums of those runs are
// joined in shared memory, the workgroups' by conv_sums_kernel, both in a fixed order.
template <typename T, int K, bool SMALL, bool STREAM>
__global__ __launch_bounds__(256) void conv_grad_kernel(ConvArgs a, T* __restrict__ dx, T* __restrict__ dstate, float* __restrict__ partial, int lx) {
    constexpr int W = 4, U = Group<K>::U;
    using P = Piece<T, W, SMALL>;
    extern __shared__ float shared[];  // [256 / lx][K + 1][W][lx]
    const int tx = threadIdx.x % lx, ty = threadIdx.x / lx, ly = 256 / lx;
    const int piece = blockIdx.x * lx + tx;
    float dw[K][W] = {}, db[W] = {};
    if (piece < a.cpr) {
        const int c = piece_start<W, SMALL>(piece, a.D);
        float w[K][W], bias[W];
        taps_of<K, W>(a, c, w, bias);
        const int64_t total = static_cast<int64_t>(a.B) * a.runs, high = static_cast<int64_t>(gridDim.y) * ly;
        for (int64_t row = static_cast<int64_t>(blockIdx.y) * ly + ty; row < total; row += high) {
            const int b = static_cast<int>(row / a.runs), r = static_cast<int>(row - static_cast<int64_t>(b) * a.runs);
            const int len = length_of(a.lengths, b, a.N), l0 = r * a.run, l1 = l0 + a.run < a.N ? l0 + a.run : a.N;
            float ring[K][W], grad[K][W];  // of position l: ring[l mod K] its input, grad[l mod K] its dpre
            Input<T, K, W, SMALL> v[U];
            P d[U];
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < W; ++j) grad[k][j] = 0.0f;
#pragma unroll
            for (int k = 1; k < K; ++k) v[k - 1].load(a, b, l0 - K + k, len, c);
#pragma unroll
            for (int k = 1; k < K; ++k) v[k - 1].get(ring[k]);
            const T* dout = static_cast<const T*>(a.dout.data) + b * a.dout.batch + c;
            T* o = dx + static_cast<int64_t>(b) * a.N * a.D + c;
            for (int l = l0; l < l1 + K - 1; l += U) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    v[u].load(a, b, l + u, len, c);
                    d[u].load(l + u < len ? dout + (l + u) * a.dout.row : reinterpret_cast<const T*>(a.weight), a.D);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float res[W], dy[W];
                    const bool in = l + u < len, own = in && l + u < l1;
                    v[u].get(ring[u % K]);
                    d[u].get(dy);
#pragma unroll
                    for (int j = 0; j < W; ++j) {
                        float pre = bias[j];
#pragma unroll
                        for (int k = 0; k < K; ++k) pre = fmaf(w[k][j], ring[(u + 1 + k) % K][j], pre);
                        const float gate = sigmoid(pre);
                        grad[u % K][j] = in ? dy[j] * gate * fmaf(pre, 1.0f - gate, 1.0f) : 0.0f;
                        float sum = 0.0f;
#pragma unroll
                        for (int k = 0; k < K; ++k) sum = fmaf(w[k][j], grad[(u + K - k) % K][j], sum);  // w[k] dpre[l - k]: of input l - K + 1
                        res[j] = sum;
                    }
                    if (own) {
#pragma unroll
                        for (int j = 0; j < W; ++j) {
                            db[j] += grad[u % K][j];
#pragma unroll
                            for (int k = 0; k < K; ++k) dw[k][j] = fmaf(grad[u % K][j], ring[(u + 1 + k) % K][j], dw[k][j]);
                        }
                    }
                    const int to = l + u - (K - 1);
                    if (to >= l0 && to < l1) {
#pragma unroll
                        for (int j = 0; j < W; ++j) res[j] = to < len ? res[j] : 0.0f;
                        P::template put<STREAM>(o + static_cast<int64_t>(to) * a.D, a.D, res);
                    } else if (r == 0 && to < 0 && dstate) {
                        P::put(dstate + (static_cast<int64_t>(b) * (K - 1) + (to + K - 1)) * a.D + c, a.D, res);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < W; ++j) {
#pragma unroll
        for (int k = 0; k < K; ++k) shared[((ty * (K + 1) + k) * W + j) * lx + tx] = dw[k][j];
        shared[((ty * (K + 1) + K) * W + j) * lx + tx] = db[j];
    }
    __syncthreads();
    const int per_run = (K + 1) * W * lx;
    for (int e = threadIdx.x; e < per_run; e += 256) {
        float sum = 0.0f;
        for (int y = 0; y < ly; ++y) sum += shared[y * per_run + e];
        const int x = e % lx, j = e / lx % W, k = e / lx / W, at = blockIdx.x * lx + x;
        const int ch = piece_start<W, SMALL>(at, a.D) + j;
        if (at < a.cpr && ch < a.D) partial[(static_cast<int64_t>(blockIdx.y) * (K + 1) + k) * a.D + ch] = sum;
    }
}

// Workgroups of 64 channels of one tap (`blocks` such in all), sixteen threads a channel over the partial sums.
template <int K>
__global__ __launch_bounds__(1024) void conv_sums_kernel(const float* __restrict__ partial, int parts, int D, int blocks, float* __restrict__ dweight,
                                                         float* __restrict__ dbias) {
    __shared__ float sums[16][64];
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6, k = blockIdx.y;
    for (int block = blockIdx.x; block < blocks; block += gridDim.x) {
        const int64_t ch = static_cast<int64_t>(block) * 64 + x;
        float sum = 0.0f;
        if (ch < D)
            for (int p = y; p < parts; p += 16) sum += partial[(static_cast<int64_t>(p) * (K + 1) + k) * D + ch];
        sums[y][x] = sum;
        __syncthreads();
        if (y == 0 && ch < D) {
            for (int i = 1; i < 16; ++i) sum += sums[i][x];
            if (k < K) dweight[ch * K + k] = sum;
            else if (dbias) dbias[ch] = sum;
        }
        __syncthreads();
    }
}

// The state moves on in place, so no two threads may share a channel: widths that are no multiple of a piece go one by one.
template <typename T, int K, int W>
__global__ __launch_bounds__(256) void conv_step_kernel(const T* __restrict__ x, int64_t x_row, ConvArgs a, T* __restrict__ state, T* __restrict__ out) {
    using P = Piece<T, W, W == 1>;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t b = id / a.cpr;
    if (b >= a.B) return;
    const int c = static_cast<int>(id - b * a.cpr) * W;
    float w[K][W], pre[W];
    P rows[K];
    T* mine = state + b * (K - 1) * a.D + c;
#pragma unroll
    for (int k = 0; k < K - 1; ++k) rows[k].load(mine + static_cast<int64_t>(k) * a.D, a.D);
    rows[K - 1].load(x + b * x_row + c, a.D);
    taps_of<K, W>(a, c, w, pre);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float v[W];
        rows[k].get(v);
#pragma unroll
        for (int j = 0; j < W; ++j) pre[j] = fmaf(w[k][j], v[j], pre[j]);
        if (k) P::put(mine + static_cast<int64_t>(k - 1) * a.D, a.D, v);
    }
#pragma unroll
    for (int j = 0; j < W; ++j) pre[j] *= sigmoid(pre[j]);
    P::put(out + b * a.D + c, a.D, pre);
}

// Positions of a run: 64, or half and half again of that while there would be fewer than `least` threads; always a multiple of the
// positions in flight, two of them at least but for five taps, whose 60 goes by 30 and 15 to 5: one.  (Held at 10 there, us 10 / 5: small forward calls
// 5.9 / 5.0, B=4 N=100 D=256, small gradients 12.1 + 3.9 / 10.4 + 3.9; B=32 N=128 D=512 9.2 / 7.8 and 13.8 + 3.8 / 14.0 + 5.0, B=2 N=4000 D=200
// 6.9 / 6.5 and 13.5 + 4.9 / 13.6 + 8.3.)  Measured: forward B=64 N=512 D=2048 bfloat16 67 us with runs of 64 (131072 threads), 72 of 32,
// 77 of 16 (what a run reads in front of it, and its taps, come to more); forward and gradient of B=128 N=128 D=1001 float, ragged, 69 us
// with 64K threads at least in the gradient (runs of 32), 79 with 128K (of 16), 73 with 32K (of 64).
int run_length(int K, int64_t threads_a_position, int N, int64_t least) {
    const int unit = K == 3 ? 6 : K == 2 ? 4 : K;
    int run = 64 / unit * unit;
    while (run > 2 * unit && threads_a_position * ((N + run - 1) / run) < least) run = run / 2 / unit * unit;
    return run;
}
constexpr int64_t kForwardThreads = 128 << 10, kGradThreads = 64 << 10;

struct GradPlan { int run, runs, lx, high; };
GradPlan grad_plan(int B, int N, int D, int K) {
    GradPlan p;
    const int cpr = pieces_of_row(D, 4);
    p.lx = 1;
    while (p.lx < 64 && p.lx < cpr) p.lx *= 2;
    p.run = run_length(K, static_cast<int64_t>(B) * cpr, N, kGradThreads);
    p.runs = (N + p.run - 1) / p.run;
    const int64_t total = static_cast<int64_t>(B) * p.runs, ly = 256 / p.lx, wide = (cpr + p.lx - 1) / p.lx;
    // at most 2048 workgroups, then they take several runs one after the other
    int64_t high = (total + ly - 1) / ly, most = 2048 / wide;
    if (most < 1) most = 1;
    if (high > most) high = most;
    p.high = static_cast<int>(high < 1 ? 1 : high);
    return p;
}

template <typename T, int K>
hipError_t conv_of(ConvArgs a, void* out, void* final_state, hipStream_t st) {
    a.cpr = pieces_of_row(a.D, Wide<T>::V);
    a.run = run_length(K, static_cast<int64_t>(a.B) * a.cpr, a.N, kForwardThreads);
    a.runs = (a.N + a.run - 1) / a.run;
    const int64_t threads = static_cast<int64_t>(a.B) * a.runs * a.cpr;
    if (!fits((threads + 255) / 256, 256)) return hipErrorInvalidValue;
    const bool stream = past_caches(static_cast<int64_t>(a.B) * a.N * a.D * static_cast<int64_t>(sizeof(T)));
    const auto kernel = a.D < Wide<T>::V ? conv_kernel<T, K, true, false> : stream ? conv_kernel<T, K, false, true> : conv_kernel<T, K, false, false>;
    kernel<<<static_cast<unsigned>((threads + 255) / 256), 256, 0, st>>>(a, static_cast<T*>(out), static_cast<T*>(final_state));
    return hipGetLastError();
}

template <typename T, int K>
hipError_t conv_grad_of(ConvArgs a, void* dx, float* dweight, float* dbias, void* dstate, void* ws, hipStream_t st) {
    const GradPlan p = grad_plan(a.B, a.N, a.D, K);
    a.cpr = pieces_of_row(a.D, 4);
    a.run = p.run;
    a.runs = p.runs;
    float* partial = static_cast<float*>(ws);
    const dim3 grid((a.cpr + p.lx - 1) / p.lx, p.high);
    const bool stream = past_caches(static_cast<int64_t>(a.B) * a.N * a.D * static_cast<int64_t>(sizeof(T)));
    const auto kernel = a.D < 4 ? conv_grad_kernel<T, K, true, false> : stream ? conv_grad_kernel<T, K, false, true> : conv_grad_kernel<T, K, false, false>;
    kernel<<<grid, 256, sizeof(float) * 256 * (K + 1) * 4, st>>>(a, static_cast<T*>(dx), static_cast<T*>(dstate), partial, p.lx);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const int blocks = pieces_of_row(a.D, 64);
    conv_sums_kernel<K><<<dim3(blocks < kColumnBlocks ? blocks : kColumnBlocks, K + 1), 1024, 0, st>>>(partial, p.high, a.D, blocks, dweight, dbias);
    return hipGetLastError();
}

template <typename T, int K>
hipError_t conv_step_of(const void* x, int64_t x_row, const float* weight, const float* bias, void* state, int B, int D, void* out, hipStream_t st) {
    const int W = D % 4 == 0 ? 4 : 1;
    const ConvArgs a{{}, {}, weight, bias, state, nullptr, B, 1, D, D / W, 0, 0};
    const int64_t blocks = (static_cast<int64_t>(B) * a.cpr + 255) / 256;
    if (!fits(blocks, 256)) return hipErrorInvalidValue;
    const auto kernel = W == 4 ? conv_step_kernel<T, K, 4> : conv_step_kernel<T, K, 1>;
    kernel<<<static_cast<unsigned>(blocks), 256, 0, st>>>(static_cast<const T*>(x), x_row, a, static_cast<T*>(state), static_cast<T*>(out));
    return hipGetLastError();
}

#define LCCRF_BY_TAPS(T, call)             \
    switch (K) {                           \
        case 2: return call(T, 2);         \
        case 3: return call(T, 3);         \
        case 4: return call(T, 4);         \
        case 5: return call(T, 5);         \
        case 6: return call(T, 6);         \
        case 7: return call(T, 7);         \
        case 8: return call(T, 8);         \
        default: return hipErrorInvalidValue; \
    }

}  // namespace

hipError_t launch_conv(int dtype, AnyRows x, const float* weight, const float* bias, const void* state, const int32_t* lengths, int B, int N, int D, int K,
                       void* out, void* final_state, hipStream_t st) {
    const ConvArgs a{x, {}, weight, bias, state, lengths, B, N, D, 0, 0, 0};
#define LCCRF_CALL(T, k) conv_of<T, k>(a, out, final_state, st)
    if (dtype) LCCRF_BY_TAPS(uint16_t, LCCRF_CALL)
    LCCRF_BY_TAPS(float, LCCRF_CALL)
#undef LCCRF_CALL
}

size_t conv_grad_workspace(int B, int N, int D, int K) {
    return up256(static_cast<size_t>(grad_plan(B, N, D, K).high) * (K + 1) * D * sizeof(float));
}

hipError_t launch_conv_grad(int dtype, AnyRows dout, AnyRows x, const float* weight, const float* bias, const void* state, const int32_t* lengths, int B, int N,
                            int D, int K, void* dx, float* dweight, float* dbias, void* dstate, void* ws, hipStream_t st) {
    const ConvArgs a{x, dout, weight, bias, state, lengths, B, N, D, 0, 0, 0};
#define LCCRF_CALL(T, k) conv_grad_of<T, k>(a, dx, dweight, dbias, dstate, ws, st)
    if (dtype) LCCRF_BY_TAPS(uint16_t, LCCRF_CALL)
    LCCRF_BY_TAPS(float, LCCRF_CALL)
#undef LCCRF_CALL
}

hipError_t launch_conv_step(int dtype, const void* x, int64_t x_row, const float* weight, const float* bias, void* state, int B, int D, int K, void* out,
                            hipStream_t st) {
#define LCCRF_CALL(T, k) conv_step_of<T, k>(x, x_row, weight, bias, state, B, D, out, st)
    if (dtype) LCCRF_BY_TAPS(uint16_t, LCCRF_CALL)
    LCCRF_BY_TAPS(float, LCCRF_CALL)
#undef LCCRF_CALL
}

}  // namespace enc
}  // namespace lccrf
