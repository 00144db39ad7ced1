// Distillation from a teacher's top logits, and its gradient.
//
// With M the largest logit, s = sum exp((x - M) / t), Mt and st the teacher's: log q_k = (v_k - Mt) / t - log st, log p = (x - M) / t - log s, so
//     loss = t sum_k q_k ((v_k - Mt) - (x[id_k] - M) + t log(s / st)),   lse = M / t + log s,   dlogits = dloss t (exp((x - M) / t) / s - q).
// The logits read (and their gradient written) are what bounds it.  Few classes: a team of lanes has a position in registers, and reads it
// once.  Many: a workgroup a position.  A row is taken in whole pieces of 16 bytes, what is left over one class a thread: no two
// threads have the same class, so the gradient may be written over the logits.
#include "lccrf_layers.h"

#include <type_traits>

namespace lccrf {
namespace enc {
namespace {

constexpr int kEntries = 4;  // of a lane, at most: LCCRF_MAX_TOP over 64
constexpr float kLeast = -3.402823466e38f;

template <int L> __device__ __forceinline__ float team_max(float v) { return max_across(v, L); }
template <int L> __device__ __forceinline__ float team_sum(float v) { return sum_across(v, L); }

// The teacher's entries of a position, entry t + e L with lane t of its team.
template <typename T, int L, int E> struct Entries {
    int id[E];    // -1: not there
    float v[E];   // its logit, then q
    float x[E];   // the student's logit
    float lead[E];  // v - Mt
    __device__ __forceinline__ void load(const DistillIn& in, int64_t row, int t, bool there) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int k = t + e * L;
            id[e] = -1;
            v[e] = -__builtin_inff();
            if (there && k < in.K) {
                const int i = in.ids[row * in.K + k];
                v[e] = in.teacher[row * in.K + k];
                id[e] = i >= 0 && i < in.V && v[e] != -__builtin_inff() ? i : -1;
            }
        }
    }
    __device__ __forceinline__ bool some() const {
        bool is = false;
#pragma unroll
        for (int e = 0; e < E; ++e) is = is || id[e] >= 0;
        return is;
    }
    __device__ __forceinline__ void gather(const T* logits) {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = id[e] >= 0 ? get1(logits + id[e]) : 0.0f;
    }
    // v becomes q; the teacher's log of its sum
    __device__ __forceinline__ float settle(float k2) {
        float top = kLeast, sum = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) top = id[e] >= 0 ? __builtin_elementwise_maximum(top, v[e]) : top;
        top = team_max<L>(top);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            lead[e] = v[e] - top;
            v[e] = id[e] >= 0 ? exp2_fast(lead[e] * k2) : 0.0f;
            sum += v[e];
        }
        sum = team_sum<L>(sum);
        const float r = 1.0f / sum;
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = id[e] >= 0 ? v[e] * r : 0.0f;
        return kLn2f * __builtin_amdgcn_logf(sum);
    }
    // The loss, M and log_s the student's.  One t is taken into the sum: differences of logits divided by a small t could pass the largest float where what is
    // left of them times t^2 does not.
    __device__ __forceinline__ float loss(float t, float log_st, float M, float log_s) const {
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) sum += v[e] == 0.0f ? 0.0f : v[e] * fmaf(log_s - log_st, t, lead[e] - (x[e] - M));
        return t * team_sum<L>(sum);
    }
    // q of every class that is named, with its first entry; that entry alone keeps its id.  K steps of one wave: rows of few classes take them only where a class is named twice
    // (team_kernel's table), rows by workgroups always, where the other waves read on meanwhile or wait.
    __device__ __forceinline__ void gather_twice(int K) {
        float all[E];
        bool first[E];
        const int lane = threadIdx.x & 63, t = lane % L, base = lane - t;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            all[e] = 0.0f;
            first[e] = id[e] >= 0;
        }
#pragma unroll
        for (int f = 0; f < E; ++f)
            for (int s = 0; s < L && f * L + s < K; ++s) {
                // (64 lanes: the entry is the same for all of them)
                const int other = L == 64 ? __builtin_amdgcn_readlane(id[f], s) : __shfl(id[f], base + s);
                const float q = L == 64 ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v[f]), s)) : __shfl(v[f], base + s);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const bool same = other == id[e];
                    all[e] += same ? q : 0.0f;
                    first[e] = first[e] && !(same && f * L + s < t + e * L);
                }
            }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            v[e] = all[e];
            if (!first[e]) id[e] = -1;
        }
    }
};

// ---- few classes: a team of L lanes a position -----------------------------------------------------------------
// R pieces of W classes a lane, and one more class with the first lanes where V is no multiple of W.  Looking for classes named twice by the table instead of comparing
// all entries with all: 46408 rows of 110 classes with 86 entries 31 us / 187, 32768 of 2000 with 64 50 / 72.
template <typename T, int L, int R, int E, bool GRAD>
__global__ __launch_bounds__(256) void team_kernel(DistillIn in, const float* __restrict__ dloss, float* __restrict__ loss, float* __restrict__ lse, T* dlogits) {
    constexpr int W = Wide<T>::V;
    const int lane = threadIdx.x & 63, t = lane % L, pieces = in.V / W, left = in.V - pieces * W;
    const float per_t = 1.0f / in.temperature, k2 = kLog2e * per_t;
    // which entry names a class: V is less than a piece more than all lanes'
    __shared__ uint8_t named[GRAD ? 256 / L : 1][GRAD ? (L * R + 1) * W : 1];
    [[maybe_unused]] uint8_t* mine = named[GRAD ? threadIdx.x / L : 0];
    const int64_t teams = static_cast<int64_t>(gridDim.x) * (256 / L);
    const int64_t rounds = (in.n + teams - 1) / teams;
    int64_t row = static_cast<int64_t>(blockIdx.x) * (256 / L) + threadIdx.x / L;
    for (int64_t round = 0; round < rounds; ++round, row += teams) {
        const bool there = row < in.n;
        const T* x0 = static_cast<const T*>(in.logits) + (there ? row : 0) * in.row;
        Entries<T, L, E> top;
        top.load(in, row, t, there);
        // of this team's lanes
        const uint64_t bits = __ballot(top.some()) >> (lane - t);
        const bool some = (L == 64 ? bits : bits & ((uint64_t{1} << (L % 64)) - 1)) != 0;
        float x[R][W], last = -__builtin_inff();
        Piece<T, W> raw[R];
        if (some) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (t + r * L < pieces) raw[r].load(x0 + (t + r * L) * W, W);
            if (t < left) last = get1(x0 + pieces * W + t);
            top.gather(x0);
        }
        float M = __builtin_elementwise_maximum(kLeast, last);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            raw[r].get(x[r]);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                x[r][j] = some && t + r * L < pieces ? x[r][j] : -__builtin_inff();
                M = __builtin_elementwise_maximum(M, x[r][j]);
            }
        }
        M = team_max<L>(M);
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < W; ++j) s += x[r][j] = exp2_fast((x[r][j] - M) * k2);
        last = exp2_fast((last - M) * k2);
        s = team_sum<L>(s + last);
        const float log_s = kLn2f * __builtin_amdgcn_logf(s), log_st = top.settle(k2);
        if (loss) {
            const float d = top.loss(in.temperature, log_st, M, log_s);
            if (there && t == 0) loss[row] = some ? d : 0.0f;
        }
        if (!GRAD && there && t == 0) lse[row] = some ? fmaf(M, per_t, log_s) : 0.0f;
        if constexpr (GRAD) {
            const float scale = there ? dloss[row] * in.temperature : 0.0f, share = 1.0f / s;
            // A class that is named once is that entry's own: of a class's entries one stays in the table, the others see it.  Comparing all with all, which costs K steps
            // a row, is for waves that have a class twice.
            bool twice = false;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (top.id[e] >= 0) mine[top.id[e]] = static_cast<uint8_t>(t + e * L);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int e = 0; e < E; ++e) twice = twice || (top.id[e] >= 0 && mine[top.id[e]] != t + e * L);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (__ballot(twice)) top.gather_twice(in.K);
            if (there) {
                T* o = dlogits + row * in.V;
#pragma unroll
                for (int r = 0; r < R; ++r) {
#pragma unroll
                    for (int j = 0; j < W; ++j) x[r][j] = some ? x[r][j] * share * scale : 0.0f;
                    if (t + r * L < pieces) Piece<T, W>::put(o + (t + r * L) * W, W, x[r]);
                }
                if (t < left) put1(o + pieces * W + t, some ? last * share * scale : 0.0f);
                // behind the same wave's stores above
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (top.id[e] >= 0) put1(o + top.id[e], (exp2_fast((top.x[e] - M) * k2) * share - top.v[e]) * scale);
            }
        }
    }
}

// ---- many classes: a workgroup a position ----------------------------------------------------------------------
template <typename T, int THREADS, int E, bool GRAD>
__global__ __launch_bounds__(THREADS) void row_kernel(DistillIn in, const float* __restrict__ dloss, const float* __restrict__ given, float* __restrict__ loss,
                                                      float* __restrict__ lse, T* dlogits) {
    constexpr int W = Wide<T>::V, kWaves = THREADS / 64, U = 4;  // pieces in flight
    __shared__ float tops[kWaves], sums[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, pieces = in.V / W, left = in.V - pieces * W;
    const float per_t = 1.0f / in.temperature, k2 = kLog2e * per_t;
    for (int64_t row = blockIdx.x; row < in.n; row += gridDim.x) {
        const T* x0 = static_cast<const T*>(in.logits) + row * in.row;
        T* o = GRAD ? dlogits + row * in.V : nullptr;
        Entries<T, 64, E> top;
        top.load(in, row, lane, true);
        if (__ballot(top.some()) == 0) {  // the same in all waves
            if (tid == 0 && loss) loss[row] = 0.0f;
            if (tid == 0 && !GRAD) lse[row] = 0.0f;
            if (GRAD) {
                const float zero[W] = {};
                for (int k = tid; k < pieces; k += THREADS) Piece<T, W>::put(o + static_cast<int64_t>(k) * W, W, zero);
                if (tid < left) put1(o + static_cast<int64_t>(pieces) * W + tid, 0.0f);
            }
            continue;
        }
        if (wave == 0) top.gather(x0);
        float M, log_s;
        if (GRAD && given) {
            M = 0.0f;
            log_s = given[row];
        } else {
            float m = kLeast, s = 0.0f;
            const auto take = [&](const Piece<T, W>& raw) {
                float x[W];
                raw.get(x);
                float now = m;
#pragma unroll
                for (int j = 0; j < W; ++j) now = __builtin_elementwise_maximum(now, x[j]);
                s *= exp2_fast((m - now) * k2);
#pragma unroll
                for (int j = 0; j < W; ++j) s += exp2_fast((x[j] - now) * k2);
                m = now;
            };
            int k = tid;
            for (; k + (U - 1) * THREADS < pieces; k += U * THREADS) {
                Piece<T, W> raw[U];
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u].load(x0 + static_cast<int64_t>(k + u * THREADS) * W, W);
#pragma unroll
                for (int u = 0; u < U; ++u) take(raw[u]);
            }
            for (; k < pieces; k += THREADS) {
                Piece<T, W> raw;
                raw.load(x0 + static_cast<int64_t>(k) * W, W);
                take(raw);
            }
            if (tid < left) {
                const float x = get1(x0 + static_cast<int64_t>(pieces) * W + tid), now = __builtin_elementwise_maximum(m, x);
                s = s * exp2_fast((m - now) * k2) + exp2_fast((x - now) * k2);
                m = now;
            }
            const float wave_top = team_max<64>(m);
            s = team_sum<64>(s * exp2_fast((m - wave_top) * k2));
            __syncthreads();
            if (lane == 0) {
                tops[wave] = wave_top;
                sums[wave] = s;
            }
            __syncthreads();
            M = tops[0];
#pragma unroll
            for (int v = 1; v < kWaves; ++v) M = __builtin_elementwise_maximum(M, tops[v]);
            s = 0.0f;
#pragma unroll
            for (int v = 0; v < kWaves; ++v) s += sums[v] * exp2_fast((tops[v] - M) * k2);
            log_s = kLn2f * __builtin_amdgcn_logf(s);
        }
        const float scale = GRAD ? dloss[row] * in.temperature : 0.0f, log2_s = kLog2e * log_s;
        if (wave == 0) {
            const float log_st = top.settle(k2);
            if (loss) {
                const float d = top.loss(in.temperature, log_st, M, log_s);
                if (lane == 0) loss[row] = d;
            }
            if (!GRAD && lane == 0) lse[row] = fmaf(M, per_t, log_s);
            if (GRAD) top.gather_twice(in.K);
        }
        if constexpr (GRAD) {
            // dlogits may be the logits: the entries' have come before any of the workgroup's stores goes out
#pragma unroll
            for (int e = 0; e < E; ++e) asm volatile("" : "+v"(top.x[e]));
            __syncthreads();
            const auto turn = [&](const Piece<T, W>& raw, int k) {
                float x[W];
                raw.get(x);
#pragma unroll
                for (int j = 0; j < W; ++j) x[j] = exp2_fast(fmaf(x[j] - M, k2, -log2_s)) * scale;
                Piece<T, W>::template put<true>(o + static_cast<int64_t>(k) * W, W, x);
            };
            int k = tid;
            for (; k + (U - 1) * THREADS < pieces; k += U * THREADS) {
                Piece<T, W> raw[U];
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u].load(x0 + static_cast<int64_t>(k + u * THREADS) * W, W);
#pragma unroll
                for (int u = 0; u < U; ++u) turn(raw[u], k + u * THREADS);
            }
            for (; k < pieces; k += THREADS) {
                Piece<T, W> raw;
                raw.load(x0 + static_cast<int64_t>(k) * W, W);
                turn(raw, k);
            }
            if (tid < left) {
                const int64_t at = static_cast<int64_t>(pieces) * W + tid;
                put1(o + at, exp2_fast(fmaf(get1(x0 + at) - M, k2, -log2_s)) * scale);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the row is written, then the named classes once more
            __syncthreads();
            if (wave == 0) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (top.id[e] >= 0) put1(o + top.id[e], (exp2_fast(fmaf(top.x[e] - M, k2, -log2_s)) - top.v[e]) * scale);
            }
        }
    }
}

// ---- many classes, loss and gradient in one: a row in registers --------------------------------------------------
// A workgroup has a row, R pieces a thread, and reads it once.  The first wave finds the named classes and leaves them in LDS, chained by the thread that has
// the class in its registers: that thread writes them once more behind its row, the difference rounded once (the classes of a chain differ, so their order does
// not matter).
struct Named { int id, next; float x, q; };
template <typename T, int THREADS, int R, int E>
__global__ __launch_bounds__(THREADS) void held_kernel(DistillIn in, const float* __restrict__ dloss, float* __restrict__ loss, T* dlogits) {
    constexpr int W = Wide<T>::V, kWaves = THREADS / 64;
    __shared__ float tops[kWaves], sums[kWaves];
    __shared__ int heads[THREADS];
    __shared__ Named named[64 * E];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), pieces = in.V / W, left = in.V - pieces * W;
    const float per_t = 1.0f / in.temperature, k2 = kLog2e * per_t;
    const int64_t row = blockIdx.x;
    const T* from = static_cast<const T*>(in.logits) + row * in.row;
    T* o = dlogits + row * in.V;
    Entries<T, 64, E> top;
    top.load(in, row, lane, true);
    if (__ballot(top.some()) == 0) {  // the same in all waves
        if (tid == 0 && loss) loss[row] = 0.0f;
        const float zero[W] = {};
        for (int k = tid; k < pieces; k += THREADS) Piece<T, W>::put(o + static_cast<unsigned>(k) * W, W, zero);
        if (tid < left) put1(o + static_cast<unsigned>(pieces) * W + tid, 0.0f);
        return;
    }
    Piece<T, W> raw[R];
    T rest{};
#pragma unroll
    for (int r = 0; r < R; ++r) {  // a thread without a piece takes the last one
        if (r * THREADS >= pieces) break;
        const unsigned k = tid + r * THREADS < pieces ? tid + r * THREADS : pieces - 1;
        raw[r].raw = *reinterpret_cast<const typename Piece<T, W>::Any*>(reinterpret_cast<const char*>(from) + k * 16u);
    }
    if (tid < left) rest = from[static_cast<unsigned>(pieces) * W + tid];
    heads[tid] = -1;
    lds_sync();
    float log_st = 0.0f;
    if (wave == 0) {
        top.gather(from);
        log_st = top.settle(k2);
        Entries<T, 64, E> once = top;
        once.gather_twice(in.K);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (once.id[e] >= 0) {
                const int piece = once.id[e] / W, owner = piece < pieces ? piece % THREADS : once.id[e] - pieces * W;
                Named& n = named[lane + e * 64];
                n.id = once.id[e];
                n.x = once.x[e];
                n.q = once.v[e];
                n.next = atomicExch(&heads[owner], lane + e * 64);
            }
    }
    float m = kLeast, s = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (r * THREADS >= pieces) break;
        float x[W];
        asm volatile("" : "+v"(raw[r].raw));  // (widened where it is used and not kept so)
        raw[r].get(x);
        float now = m, sum = 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) now = __builtin_elementwise_maximum(now, x[j]);
#pragma unroll
        for (int j = 0; j < W; ++j) sum += exp2_fast((x[j] - now) * k2);
        // (the last piece once more: its maximum does no harm)
        s = fmaf(s, exp2_fast((m - now) * k2), tid + r * THREADS < pieces ? sum : 0.0f);
        m = now;
        __builtin_amdgcn_sched_barrier(0);
    }
    if (tid < left) {
        const float x = widen(rest), now = __builtin_elementwise_maximum(m, x);
        s = s * exp2_fast((m - now) * k2) + exp2_fast((x - now) * k2);
        m = now;
    }
    const float wave_top = team_max<64>(m);
    s = team_sum<64>(s * exp2_fast((m - wave_top) * k2));
    if (lane == 0) {
        tops[wave] = wave_top;
        sums[wave] = s;
    }
    // dlogits may be the logits: what the loss reads of the named classes has come before any of the workgroup's stores goes out.  (The barrier orders LDS alone, and
    // a slot whose entries all name classes again has left nothing there.)
    if (wave == 0) {
#pragma unroll
        for (int e = 0; e < E; ++e) asm volatile("" : "+v"(top.x[e]));
    }
    lds_sync();
    float M = tops[0];
#pragma unroll
    for (int v = 1; v < kWaves; ++v) M = __builtin_elementwise_maximum(M, tops[v]);
    s = 0.0f;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) s += sums[v] * exp2_fast((tops[v] - M) * k2);
    const float scale = dloss[row] * in.temperature, share = scale / s;
    if (wave == 0 && loss) {
        const float d = top.loss(in.temperature, log_st, M, kLn2f * __builtin_amdgcn_logf(s));
        if (lane == 0) loss[row] = d;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (r * THREADS >= pieces) break;
        float x[W];
        asm volatile("" : "+v"(raw[r].raw));
        raw[r].get(x);
#pragma unroll
        for (int j = 0; j < W; ++j) x[j] = exp2_fast((x[j] - M) * k2) * share;
        if (tid + r * THREADS < pieces) Piece<T, W>::template put<true>(o + static_cast<unsigned>(tid + r * THREADS) * W, W, x);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (tid < left) put1(o + static_cast<unsigned>(pieces) * W + tid, exp2_fast((widen(rest) - M) * k2) * share);
    for (int k = heads[tid]; k >= 0;) {  // behind this thread's own stores
        const Named n = named[k];
        put1(o + n.id, fmaf(exp2_fast((n.x - M) * k2), share, -n.q * scale));
        k = n.next;
    }
}

// ---- launches -------------------------------------------------------------------------------------------------

constexpr int64_t kMostBlocks = 1 << 20;

// Measured, us, bfloat16: up to 256 pieces by teams / by workgroups, 32768 rows of 500 classes 16 / 40, 1000 18 / 35, 2000 28 / 46 (4.7 TB/s), with the gradient 1000 30 / 56,
// 2000 47 / 79 (5.6).  Loss and gradient of a row in registers / read twice: 8192 rows of 5003 39 / 47, 30000 195 / 215 (5.0), 4096 rows of 100003 389 / 468 (4.2; ragged
// lengths 357).  25 pieces a thread take 128 registers, the last that leave room for two workgroups a CU, 32 take 156: 2048 rows of 100003 196 / 229, of 70001 133 / 155; with
// more than 64 entries there is room for one either way (270 / 270), and 32 serve them all.  Read twice or the loss alone, by 256 threads / by 512: 8192 rows of
// 10000 32 / 45 (5.1), 30000 87 / 83 (5.9).

template <typename T, bool GRAD>
hipError_t distill_of(const DistillIn& in, const float* dloss, const float* given, float* loss, float* lse, void* dlogits, hipStream_t st) {
    constexpr int W = Wide<T>::V;
    const int pieces = in.V / W, wide = pieces > in.K ? pieces : in.K;
    T* o = static_cast<T*>(dlogits);
    if (pieces <= 256) {
        const auto go = [&](auto kernel, int L) {
            const int64_t blocks = (in.n + 256 / L - 1) / (256 / L);
            kernel<<<static_cast<unsigned>(blocks < kMostBlocks ? blocks : kMostBlocks), 256, 0, st>>>(in, dloss, loss, lse, o);
            return hipGetLastError();
        };
        if (in.K > 64) return go(pieces <= 64 ? team_kernel<T, 64, 1, kEntries, GRAD> : team_kernel<T, 64, 4, kEntries, GRAD>, 64);
        if (wide <= 8) return go(team_kernel<T, 8, 1, 1, GRAD>, 8);  // eight lanes: what is left over of a row has one each
        if (wide <= 16) return go(team_kernel<T, 16, 1, 1, GRAD>, 16);
        if (wide <= 32) return go(team_kernel<T, 32, 1, 1, GRAD>, 32);
        if (wide <= 64) return go(team_kernel<T, 64, 1, 1, GRAD>, 64);
        return go(wide <= 128 ? team_kernel<T, 64, 2, 1, GRAD> : team_kernel<T, 64, 4, 1, GRAD>, 64);
    }
    const bool many = in.K > 64;
    if constexpr (GRAD) {
        if (!given && pieces <= 16384 && in.n < kMostBlocks) {
            const auto go = [&](auto kernel, int threads) {
                kernel<<<static_cast<unsigned>(in.n), threads, 0, st>>>(in, dloss, loss, o);
                return hipGetLastError();
            };
            if (pieces <= 1024) return go(many ? held_kernel<T, 256, 4, kEntries> : held_kernel<T, 256, 4, 1>, 256);
            if (pieces <= 2048) return go(many ? held_kernel<T, 256, 8, kEntries> : held_kernel<T, 256, 8, 1>, 256);
            if (pieces <= 4096) return go(many ? held_kernel<T, 512, 8, kEntries> : held_kernel<T, 512, 8, 1>, 512);
            if (pieces <= 8192) return go(many ? held_kernel<T, 512, 16, kEntries> : held_kernel<T, 512, 16, 1>, 512);
            if (pieces <= 12800 && !many) return go(held_kernel<T, 512, 25, 1>, 512);
            return go(many ? held_kernel<T, 512, 32, kEntries> : held_kernel<T, 512, 32, 1>, 512);
        }
    }
    const unsigned blocks = static_cast<unsigned>(in.n < kMostBlocks ? in.n : kMostBlocks);
    if (pieces < 2048) {
        const auto kernel = many ? row_kernel<T, 256, kEntries, GRAD> : row_kernel<T, 256, 1, GRAD>;
        kernel<<<blocks, 256, 0, st>>>(in, dloss, given, loss, lse, o);
    } else {
        const auto kernel = many ? row_kernel<T, 512, kEntries, GRAD> : row_kernel<T, 512, 1, GRAD>;
        kernel<<<blocks, 512, 0, st>>>(in, dloss, given, loss, lse, o);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_distill(int dtype, const DistillIn& in, float* loss, float* lse, hipStream_t st) {
    return dtype ? distill_of<uint16_t, false>(in, nullptr, nullptr, loss, lse, nullptr, st) : distill_of<float, false>(in, nullptr, nullptr, loss, lse, nullptr, st);
}

hipError_t launch_distill_grad(int dtype, const float* dloss, const DistillIn& in, const float* lse, float* loss, void* dlogits, hipStream_t st) {
    return dtype ? distill_of<uint16_t, true>(in, dloss, lse, loss, nullptr, dlogits, st) : distill_of<float, true>(in, dloss, lse, loss, nullptr, dlogits, st);
}

}  // namespace enc
}  // namespace lccrf
