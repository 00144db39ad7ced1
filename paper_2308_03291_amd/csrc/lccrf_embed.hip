// Embedding lookup and its gradient.
//
// Lookup: a copy with a product.  Threads are numbered over (position, 16-byte piece of its row); what bounds it is the
// traffic of the written rows and of the distinct rows read.
//
// Gradient: rows of the table are sums over the positions that hold their token.  Adding rows where they fall would need
// atomics (an order that changes from run to run) and a float copy of the table; instead the positions are sorted by token:
//   1. index: a workgroup owns a range of tokens.  It passes over all ids twice (they stay in the caches), counts
//      and places the positions of its own tokens, and so knows without any other workgroup where they start.
//      Each of its waves has a share of the positions and its own counters, so the order is fixed.
//   2. rows: every row of the gradient by the threads of its 16-byte pieces: its positions summed in registers, or zeros.
//      Tokens with more than kPiece positions (in text a few hold a tenth of all) are cut into the pieces of kPiece sorted
//      positions that they reach into, one partial sum each.
//   3. join: those partial sums, in order.
#include "lccrf_encoder.h"

namespace lccrf {
namespace enc {
namespace {

constexpr int kItems = 4;  // pieces a thread of the lookup

template <typename T, bool SMALL>
__global__ __launch_bounds__(256) void embed_kernel(const T* __restrict__ table, int V, int D, int64_t table_row, const int32_t* __restrict__ ids,
                                                    int64_t n, float scale, T* __restrict__ out, int cpr, int per_block) {
    constexpr int W = Wide<T>::V;
    using P = Piece<T, W, SMALL>;
    // A workgroup has per_block positions (cpr pieces each); thread t the pieces t, t + 256, ...
    const int64_t first = static_cast<int64_t>(blockIdx.x) * per_block;
    const int here = static_cast<int>(n - first < per_block ? n - first : per_block) * cpr;
    for (int k0 = threadIdx.x; k0 < here; k0 += 256 * kItems) {
        int c[kItems], id[kItems];
        int64_t pos[kItems];
        P v[kItems];
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int k = k0 + 256 * i < here ? k0 + 256 * i : k0;
            const int p = k / cpr;
            c[i] = piece_start<W, SMALL>(k - p * cpr, D);
            pos[i] = first + p;
            id[i] = ids[pos[i]];
        }
#pragma unroll
        for (int i = 0; i < kItems; ++i) v[i].load(table + (static_cast<unsigned>(id[i]) < static_cast<unsigned>(V) ? id[i] * table_row : 0) + c[i], D);
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            float o[W];
            v[i].get(o);
#pragma unroll
            for (int j = 0; j < W; ++j) o[j] = static_cast<unsigned>(id[i]) < static_cast<unsigned>(V) ? o[j] * scale : 0.0f;
            if (k0 + 256 * i < here) P::put(out + pos[i] * D + c[i], D, o);
        }
    }
}

// ---- gradient -------------------------------------------------------------------------------------------------

constexpr int kIndexWaves = 16, kIndexThreads = 64 * kIndexWaves;
constexpr int kMaxRange = kIndexThreads;  // tokens of a workgroup of `index`: one a thread
constexpr int kPiece = 32;                // sorted positions a partial sum covers at most

struct IndexPlan { int range, workgroups; };
// 256 workgroups, one a compute unit, as long as their ranges hold 64 tokens at least and kMaxRange at most.
__host__ inline IndexPlan index_plan(int V) {
    int range = (V + 255) / 256;
    range = range < 64 ? 64 : range > kMaxRange ? kMaxRange : range;
    return {range, (V + range - 1) / range};
}

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_any __attribute__((aligned(4)));

// Four ids from p on; -1 past the end of the share.
__device__ __forceinline__ void four_ids(const int32_t* __restrict__ ids, int p, int end, int (&id)[4]) {
    if (p + 4 <= end) {
        const i32x4 v = *reinterpret_cast<const i32x4_any*>(ids + p);
        id[0] = v[0]; id[1] = v[1]; id[2] = v[2]; id[3] = v[3];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) id[i] = p + i < end ? ids[p + i] : -1;
    }
}

__global__ __launch_bounds__(kIndexThreads) void index_kernel(const int32_t* __restrict__ ids, int n, int V, int range, int32_t* __restrict__ order,
                                                              int32_t* __restrict__ start) {
    extern __shared__ int32_t count[];  // [kIndexWaves][range]
    __shared__ int32_t wave_sum[kIndexWaves], below_sum[kIndexWaves];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    const int lo = blockIdx.x * range, hi = lo + range < V ? lo + range : V;
    for (int k = t; k < kIndexWaves * range; k += kIndexThreads) count[k] = 0;
    __syncthreads();
    int32_t* mine = count + w * range;
    const int share = ((n + kIndexWaves - 1) / kIndexWaves + 255) / 256 * 256;
    const int64_t begin64 = static_cast<int64_t>(w) * share;
    const int begin = begin64 < n ? static_cast<int>(begin64) : n;
    const int end = begin64 + share < n ? static_cast<int>(begin64 + share) : n;
    int below = 0;
    for (int p = begin + 4 * lane; p < end; p += 256) {
        int id[4];
        four_ids(ids, p, end, id);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (id[i] >= lo && id[i] < hi) atomicAdd(&mine[id[i] - lo], 1);
            below += id[i] >= 0 && id[i] < lo;
        }
    }
    for (int d = 1; d < 64; d *= 2) below += __shfl_xor(below, d);
    if (lane == 0) below_sum[w] = below;
    __syncthreads();
    // Thread t: token lo + t.  Where its positions start, and within them those of every wave's share.
    int total = 0;
    if (t < range)
        for (int k = 0; k < kIndexWaves; ++k) total += count[k * range + t];
    int upto = total;
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 63) wave_sum[w] = upto;
    __syncthreads();
    int base = upto - total;
    for (int k = 0; k < kIndexWaves; ++k) base += below_sum[k] + (k < w ? wave_sum[k] : 0);
    if (t < range) {
        if (lo + t < V) start[lo + t] = base;
        if (lo + t == V - 1) start[V] = base + total;
        for (int k = 0; k < kIndexWaves; ++k) {
            const int here = count[k * range + t];
            count[k * range + t] = base;
            base += here;
        }
    }
    __syncthreads();
    for (int p0 = begin; p0 < end; p0 += 256) {
        const int p = p0 + 4 * lane;
        int id[4];
        four_ids(ids, p, end, id);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = id[i] >= lo && id[i] < hi;
            uint64_t left = __ballot(in);
            while (left) {
                const int leader = __builtin_ctzll(left);
                const int which = __builtin_amdgcn_readlane(id[i], leader);
                const bool same = in && id[i] == which;
                const uint64_t all = __ballot(same);
                int at = 0;
                if (lane == leader) at = atomicAdd(&mine[which - lo], __popcll(all));
                at = __builtin_amdgcn_readlane(at, leader);
                if (same) order[at + __popcll(all & ((1ull << lane) - 1))] = p + i;
                left &= ~all;
            }
        }
    }
}

struct GradArgs {
    const int32_t *ids, *order, *start;
    int n, N, V, D, cpr;
    float scale;
    float* partial;  // [pieces][2][D]
};

template <typename T, int W, bool SMALL>
__device__ __forceinline__ void sum_rows(const GradArgs& a, Rows<T> dout, int from, int to, int c, float (&sum)[W]) {
    constexpr int U = 4;
#pragma unroll
    for (int j = 0; j < W; ++j) sum[j] = 0.0f;
    for (int k = from; k < to; k += U) {
        Piece<T, W, SMALL> v[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int p = a.order[k + i < to ? k + i : k], b = p / a.N;
            v[i].load(dout.data + b * dout.batch + (p - b * a.N) * dout.row + c, a.D);
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            float o[W];
            v[i].get(o);
#pragma unroll
            for (int j = 0; j < W; ++j) sum[j] += k + i < to ? o[j] : 0.0f;
        }
    }
}

// The first `piece_blocks` workgroups: partial sums of long rows.  Slot 0 of piece j is for the row that its first
// position belongs to, slot 1 for the one of its last position, if that is another: a row of more than kPiece positions
// reaches over an end of every piece it has a part in.
template <typename T, bool SMALL>
__global__ __launch_bounds__(256) void rows_kernel(GradArgs a, Rows<T> dout, T* __restrict__ grad, int piece_blocks) {
    constexpr int W = Wide<T>::V;
    float sum[W];
    if (static_cast<int>(blockIdx.x) < piece_blocks) {
        const int64_t k = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
        const int64_t item = k / a.cpr;
        const int c = piece_start<W, SMALL>(static_cast<int>(k - item * a.cpr), a.D), slot = static_cast<int>(item & 1);
        const int64_t from64 = (item >> 1) * kPiece;
        const int total = a.start[a.V];
        if (from64 >= total) return;
        const int from = static_cast<int>(from64), to = total - from < kPiece ? total : from + kPiece;
        const int first = a.ids[a.order[from]], last = a.ids[a.order[to - 1]];
        const int row = slot ? last : first;
        if (slot && first == last) return;
        const int s = a.start[row], e = a.start[row + 1];
        if (e - s <= kPiece) return;
        sum_rows<T, W, SMALL>(a, dout, s > from ? s : from, e < to ? e : to, c, sum);
        Piece<float, W, SMALL>::put(a.partial + item * a.D + c, a.D, sum);
        return;
    }
    const int64_t k = static_cast<int64_t>(blockIdx.x - piece_blocks) * 256 + threadIdx.x;
    const int64_t row = k / a.cpr;
    if (row >= a.V) return;
    const int c = piece_start<W, SMALL>(static_cast<int>(k - row * a.cpr), a.D);
    const int s = a.start[row], e = a.start[row + 1];
    if (e - s > kPiece) return;
    sum_rows<T, W, SMALL>(a, dout, s, e, c, sum);
#pragma unroll
    for (int j = 0; j < W; ++j) sum[j] *= a.scale;
    Piece<T, W, SMALL>::put(grad + row * a.D + c, a.D, sum);
}

// A long row is joined by the threads of the piece that it begins in (it is the row of that piece's last position).
template <typename T, bool SMALL>
__global__ __launch_bounds__(256) void join_kernel(GradArgs a, T* __restrict__ grad) {
    constexpr int W = Wide<T>::V;
    const int64_t k = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t j = k / a.cpr;
    const int c = piece_start<W, SMALL>(static_cast<int>(k - j * a.cpr), a.D);
    const int64_t from = j * kPiece;
    const int total = a.start[a.V];
    if (from >= total) return;
    const int64_t to = from + kPiece < total ? from + kPiece : total;
    const int row = a.ids[a.order[to - 1]];
    const int s = a.start[row], e = a.start[row + 1];
    if (e - s <= kPiece || s < from) return;
    const int64_t last = (e - 1) / kPiece;
    float sum[W], v[W];
    Piece<float, W, SMALL> part;
    part.load(a.partial + (2 * j + (s > from)) * a.D + c, a.D);
    part.get(sum);
    for (int64_t q = j + 1; q <= last; ++q) {
        part.load(a.partial + 2 * q * a.D + c, a.D);
        part.get(v);
#pragma unroll
        for (int i = 0; i < W; ++i) sum[i] += v[i];
    }
#pragma unroll
    for (int i = 0; i < W; ++i) sum[i] *= a.scale;
    Piece<T, W, SMALL>::put(grad + static_cast<int64_t>(row) * a.D + c, a.D, sum);
}

inline int64_t pieces_of(int64_t n) { return (n + kPiece - 1) / kPiece; }

template <typename T, bool SMALL>
hipError_t embed_of(const void* table, int V, int D, int64_t table_row, const int32_t* ids, int64_t n, float scale, void* out, hipStream_t st) {
    const int cpr = (D + Wide<T>::V - 1) / Wide<T>::V;
    // positions a workgroup: its threads' kItems pieces, one position at least
    const int per_block = cpr >= 256 * kItems ? 1 : 256 * kItems / cpr;
    if (!fits((n + per_block - 1) / per_block, 256)) return hipErrorInvalidValue;
    embed_kernel<T, SMALL><<<static_cast<unsigned>((n + per_block - 1) / per_block), 256, 0, st>>>(static_cast<const T*>(table), V, D, table_row, ids, n, scale,
                                                                                           static_cast<T*>(out), cpr, per_block);
    return hipGetLastError();
}

template <typename T, bool SMALL>
hipError_t embed_grad_of(AnyRows dout, const int32_t* ids, int B, int N, int V, int D, float scale, void* grad, void* ws, hipStream_t st) {
    const int n = B * N;
    const IndexPlan plan = index_plan(V);
    char* base = static_cast<char*>(ws);
    int32_t* start = reinterpret_cast<int32_t*>(base);
    int32_t* order = reinterpret_cast<int32_t*>(base + up256((static_cast<size_t>(V) + 1) * 4));
    float* partial = reinterpret_cast<float*>(base + up256((static_cast<size_t>(V) + 1) * 4) + up256(static_cast<size_t>(n) * 4));
    const int cpr = (D + Wide<T>::V - 1) / Wide<T>::V;
    const GradArgs a{ids, order, start, n, N < 1 ? 1 : N, V, D, cpr, scale, partial};
    const int64_t pieces = n > kPiece ? pieces_of(n) : 0;  // without a row that can be long there is nothing to cut
    const int64_t piece_blocks = (2 * pieces * cpr + 255) / 256;
    const int64_t row_blocks = (static_cast<int64_t>(V) * cpr + 255) / 256;
    if (!fits(piece_blocks + row_blocks, 256)) return hipErrorInvalidValue;
    index_kernel<<<plan.workgroups, kIndexThreads, sizeof(int32_t) * kIndexWaves * plan.range, st>>>(ids, n, V, plan.range, order, start);
    rows_kernel<T, SMALL><<<static_cast<unsigned>(piece_blocks + row_blocks), 256, 0, st>>>(a, dout.as<T>(), static_cast<T*>(grad), static_cast<int>(piece_blocks));
    if (pieces) join_kernel<T, SMALL><<<static_cast<unsigned>((pieces * cpr + 255) / 256), 256, 0, st>>>(a, static_cast<T*>(grad));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(int dtype, const void* table, int V, int D, int64_t table_row, const int32_t* ids, int64_t n, float scale, void* out, hipStream_t st) {
    if (n == 0) return hipSuccess;
    const auto of = dtype ? (D < Wide<uint16_t>::V ? embed_of<uint16_t, true> : embed_of<uint16_t, false>) : (D < Wide<float>::V ? embed_of<float, true> : embed_of<float, false>);
    return of(table, V, D, table_row, ids, n, scale, out, st);
}

size_t embed_grad_workspace(int64_t n, int V, int D) {
    return up256((static_cast<size_t>(V) + 1) * 4) + up256(static_cast<size_t>(n) * 4) + up256(n > kPiece ? static_cast<size_t>(pieces_of(n)) * 2 * D * 4 : 0) + 256;
}

hipError_t launch_embed_grad(int dtype, AnyRows dout, const int32_t* ids, int B, int N, int V, int D, float scale, void* grad, void* ws, hipStream_t st) {
    const auto of = dtype ? (D < Wide<uint16_t>::V ? embed_grad_of<uint16_t, true> : embed_grad_of<uint16_t, false>)
                          : (D < Wide<float>::V ? embed_grad_of<float, true> : embed_grad_of<float, false>);
    return of(dout, ids, B, N, V, D, scale, grad, ws, st);
}

}  // namespace enc
}  // namespace lccrf
