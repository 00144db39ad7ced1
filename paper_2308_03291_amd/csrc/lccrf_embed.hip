// Embedding lookup and its gradient.
//
// Lookup: a copy with a product.  Threads are numbered over (position, 16-byte piece of its row); what bounds it is the
// traffic of the written rows and of the distinct rows read (32768 positions of 1024 bfloat16, 102 MB: 13.8 us; a part of it stays in
// the memory-side cache).  Four pieces a thread, so that four rows are on their way at once.
//
// Gradient: rows of the table are sums over the positions that hold their token.  Adding rows where they fall would need
// atomics (an order that changes from run to run) and a float copy of the table; instead the positions are sorted by token:
//   1. index: a workgroup owns a range of tokens.  It passes over all ids (they stay in the caches), counts the positions of
//      its own tokens and those of lower ones, and so knows without any other workgroup where its own start; then it places
//      them.  Each of its waves has a share of the positions and its own counters, so the order is fixed.
//   2. rows: every row of the gradient by the threads of its 16-byte pieces: its positions summed in registers, or zeros.
//      Tokens with more than `piece` positions (in text a few hold a tenth of all) are cut into the pieces of `piece` sorted
//      positions that they reach into, one partial sum each.
//   3. join: those partial sums, in order.
// The traffic of the gradients read and of the table written is what bounds it: 32768 positions of 1024 bfloat16 into 100003 rows, 272 MB, 59 us
// (index 10.7, rows 46.0, join 4.9); small ones are bound by their three launches (2048 positions of 301 floats, 16 us).  Every workgroup of the
// index reads all ids: with many positions of narrow rows it costs most (1048576 of 32 floats into 50000 rows 71 us, the rows 28).
#include "lccrf_encoder.h"

#include <type_traits>

namespace lccrf {
namespace enc {
namespace {

constexpr int kItems = 4;  // pieces a thread of the lookup

template <typename T, bool SMALL, bool STREAM>
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
            if (k0 + 256 * i < here) P::template put<STREAM>(out + pos[i] * D + c[i], D, o);
        }
    }
}

// ---- gradient -------------------------------------------------------------------------------------------------

constexpr int kIndexWaves = 16, kIndexThreads = 64 * kIndexWaves;
constexpr int kMaxRange = kIndexThreads;  // tokens of a workgroup of `index`: one a thread
constexpr int kFlight = 8;                // loads of four ids in flight a thread: all of its share up to 32768 positions
constexpr int kKept = 1024;               // positions a wave of `index` keeps from its first pass; with more it passes over the ids again
constexpr int kRangeBits = 10;            // a kept word: position within the share and, in the lowest bits, token within the range
static_assert(kMaxRange == 1 << kRangeBits, "");

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

// This workgroup's share of `bytes` zeros from p on (elements of two bytes and more): 16-byte pieces, one a thread in turn over
// the whole launch, so that the chip writes one place after the other; the ends, by twos, are the first workgroup's.
__device__ __forceinline__ void clear(char* p, int64_t bytes, int t) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    int64_t head = -reinterpret_cast<intptr_t>(p) & 15;
    if (head > bytes) head = bytes;
    const int64_t pieces = (bytes - head) / 16, tail = bytes - head - pieces * 16;
    u32x4* const whole = reinterpret_cast<u32x4*>(p + head);
    const int64_t all = static_cast<int64_t>(gridDim.x) * kIndexThreads;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kIndexThreads + t; i < pieces; i += all) __builtin_nontemporal_store(u32x4{}, whole + i);
    if (blockIdx.x == 0) {
        if (2 * t < head) reinterpret_cast<uint16_t*>(p)[t] = 0;
        if (2 * t < tail) reinterpret_cast<uint16_t*>(whole + pieces)[t] = 0;
    }
}

// zero: the table's gradient of zero_bytes, which this launch clears as well; or null.  Workgroups behind the last range have only that to do.
__global__ __launch_bounds__(kIndexThreads) void index_kernel(const int32_t* __restrict__ ids, int n, int V, int range, int32_t* __restrict__ order,
                                                              int32_t* __restrict__ start, char* __restrict__ zero, int64_t zero_bytes) {
    extern __shared__ int32_t lds[];  // counters [kIndexWaves][range], then kept positions with their tokens [kIndexWaves][kKept]
    __shared__ int32_t wave_sum[kIndexWaves], below_sum[kIndexWaves];
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
    if (static_cast<int64_t>(blockIdx.x) * range >= V) {
        clear(zero, zero_bytes, t);
        return;
    }
    const int lo = blockIdx.x * range, hi = lo + range < V ? lo + range : V;
    const unsigned here = hi - lo;
    int32_t* const count = lds;
    uint32_t* const keep = reinterpret_cast<uint32_t*>(lds + kIndexWaves * range) + w * kKept;
    for (int k = t; k < kIndexWaves * range; k += kIndexThreads) count[k] = 0;
    __syncthreads();
    int32_t* mine = count + w * range;
    const uint64_t before = (1ull << lane) - 1;
    const int share = ((n + kIndexWaves - 1) / kIndexWaves + 255) / 256 * 256;
    const int64_t begin64 = static_cast<int64_t>(w) * share;
    const int begin = begin64 < n ? static_cast<int>(begin64) : n;
    const int end = begin64 + share < n ? static_cast<int>(begin64 + share) : n;
    int below = 0, kept = 0;
    const auto look = [&](const int (&id)[4], int p) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned local = id[i] - lo;
            below += static_cast<unsigned>(id[i]) < static_cast<unsigned>(lo);
            const bool in = local < here;
            const uint64_t all = __ballot(in);
            if (all) {  // about one id in 256 is this workgroup's
                const int to = kept + __popcll(all & before);
                if (in) {
                    atomicAdd(&mine[local], 1);
                    if (to < kKept) keep[to] = static_cast<uint32_t>(p + i - begin) << kRangeBits | local;
                }
                kept += __popcll(all);
            }
        }
    };
    int p0 = begin;
    for (; p0 + 256 * kFlight <= end; p0 += 256 * kFlight) {  // whole batches: all loads in flight, nothing to pick
        i32x4 v[kFlight];
#pragma unroll
        for (int f = 0; f < kFlight; ++f) v[f] = *reinterpret_cast<const i32x4_any*>(ids + p0 + 256 * f + 4 * lane);
#pragma unroll
        for (int f = 0; f < kFlight; ++f) {
            const int id[4] = {v[f][0], v[f][1], v[f][2], v[f][3]};
            look(id, p0 + 256 * f + 4 * lane);
        }
    }
    for (; p0 < end; p0 += 256) {
        int id[4];
        four_ids(ids, p0 + 4 * lane, end, id);
        look(id, p0 + 4 * lane);
    }
    for (int d = 1; d < 64; d *= 2) below += __shfl_xor(below, d);
    if (lane == 0) below_sum[w] = below;
    __syncthreads();
    // Thread t: token lo + t.  Where its positions start, and within them those of every wave's share.
    int total = 0, of_wave[kIndexWaves];
#pragma unroll
    for (int k = 0; k < kIndexWaves; ++k) {
        of_wave[k] = t < range ? count[k * range + t] : 0;
        total += of_wave[k];
    }
    int upto = total;
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 63) wave_sum[w] = upto;
    __syncthreads();
    int base = upto - total;
#pragma unroll
    for (int k = 0; k < kIndexWaves; ++k) base += below_sum[k] + (k < w ? wave_sum[k] : 0);
    if (t < range) {
        if (lo + t < V) start[lo + t] = base;
        if (lo + t == V - 1) start[V] = base + total;
#pragma unroll
        for (int k = 0; k < kIndexWaves; ++k) {
            count[k * range + t] = base;
            base += of_wave[k];
        }
    }
    __syncthreads();
    // Places: which lanes have the same token follows from one ballot a bit of it; they take theirs together.
    int bits = 0;
    while (range > 1 << bits) ++bits;
    const auto place = [&](bool in, int local, int p) {
        uint64_t same = __ballot(in);
        if (!same) return;
        for (int k = 0; k < bits; ++k) {
            const uint64_t set = __ballot(local >> k & 1);
            same &= local >> k & 1 ? set : ~set;
        }
        int at = 0;
        if (in) {
            at = mine[local];
            order[at + __popcll(same & before)] = p;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (in && !(same & before)) mine[local] = at + __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    if (kept <= kKept && share <= 1 << (32 - kRangeBits)) {
        for (int k = 0; k < kept; k += 64) {
            const bool in = k + lane < kept;
            const uint32_t v = in ? keep[k + lane] : 0;
            place(in, v & (kMaxRange - 1), begin + static_cast<int>(v >> kRangeBits));
        }
    } else {  // many of one token: all ids once more, in the same order
        for (int p0 = begin; p0 < end; p0 += 256) {
            int id[4];
            four_ids(ids, p0 + 4 * lane, end, id);
#pragma unroll
            for (int i = 0; i < 4; ++i) place(static_cast<unsigned>(id[i] - lo) < here, id[i] - lo, p0 + 4 * lane + i);
        }
    }
    if (zero) clear(zero, zero_bytes, t);
}

struct GradArgs {
    const int32_t *ids, *order, *start;
    int n, N, V, D, cpr, piece;
    float scale;
    float* partial;  // [pieces][2][D]
};

template <typename T, int W, bool SMALL>
__device__ __forceinline__ void sum_rows(const GradArgs& a, Rows<T> dout, int from, int to, int c, float (&sum)[W]) {
#pragma unroll
    for (int j = 0; j < W; ++j) sum[j] = 0.0f;
    const auto some = [&](auto many, int k) {  // that many positions, their loads in flight together
        constexpr int U = decltype(many)::value;
        Piece<T, W, SMALL> v[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int p = a.order[k + i], b = p / a.N;
            v[i].load(dout.data + b * dout.batch + (p - b * a.N) * dout.row + c, a.D);
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            float o[W];
            v[i].get(o);
#pragma unroll
            for (int j = 0; j < W; ++j) sum[j] += o[j];
        }
    };
    int k = from;
    for (; k + 8 <= to; k += 8) some(std::integral_constant<int, 8>{}, k);
    if (k + 4 <= to) { some(std::integral_constant<int, 4>{}, k); k += 4; }
    if (k + 2 <= to) { some(std::integral_constant<int, 2>{}, k); k += 2; }
    if (k < to) some(std::integral_constant<int, 1>{}, k);
}

// The first `piece_blocks` workgroups: partial sums of long rows.  Slot 0 of piece j is for the row that its first
// position belongs to, slot 1 for the one of its last position, if that is another: a row of more than `piece` positions
// reaches over an end of every piece it has a part in.  The others: ROWS rows a thread, or with ROWS = 0, where the rows are cleared
// already, the row that begins at a sorted position, if one does.
template <typename T, bool SMALL, int ROWS, bool STREAM>
__global__ __launch_bounds__(256) void rows_kernel(GradArgs a, Rows<T> dout, T* __restrict__ grad, int piece_blocks) {
    constexpr int W = Wide<T>::V;
    float sum[W];
    if (static_cast<int>(blockIdx.x) < piece_blocks) {
        const int64_t k = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
        const int64_t item = k / a.cpr;
        const int c = piece_start<W, SMALL>(static_cast<int>(k - item * a.cpr), a.D), slot = static_cast<int>(item & 1);
        const int64_t from64 = (item >> 1) * a.piece;
        const int total = a.start[a.V];
        if (from64 >= total) return;
        const int from = static_cast<int>(from64), to = total - from < a.piece ? total : from + a.piece;
        const int first = a.ids[a.order[from]], last = a.ids[a.order[to - 1]];
        const int row = slot ? last : first;
        if (slot && first == last) return;
        const int s = a.start[row], e = a.start[row + 1];
        if (e - s <= a.piece) return;
        sum_rows<T, W, SMALL>(a, dout, s > from ? s : from, e < to ? e : to, c, sum);
        Piece<float, W, SMALL>::put(a.partial + item * a.D + c, a.D, sum);
        return;
    }
    const int64_t k = static_cast<int64_t>(blockIdx.x - piece_blocks) * 256 + threadIdx.x;
    const int c = piece_start<W, SMALL>(static_cast<int>(k % a.cpr), a.D);
    if constexpr (ROWS == 0) {
        const int64_t from = k / a.cpr;
        if (from >= a.start[a.V]) return;
        const int row = a.ids[a.order[from]], s = a.start[row], e = a.start[row + 1];
        if (s != from || e - s > a.piece) return;
        sum_rows<T, W, SMALL>(a, dout, s, e, c, sum);
#pragma unroll
        for (int j = 0; j < W; ++j) sum[j] *= a.scale;
        Piece<T, W, SMALL>::template put<STREAM>(grad + static_cast<int64_t>(row) * a.D + c, a.D, sum);
        return;
    }
    const int64_t row0 = k / a.cpr * ROWS;
    if (row0 >= a.V) return;
    int s[ROWS + 1];
#pragma unroll
    for (int i = 0; i <= ROWS; ++i) s[i] = a.start[row0 + i < a.V ? row0 + i : a.V];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int n = s[i + 1] - s[i];
        if (row0 + i >= a.V || n > a.piece) continue;
        if (n) {
            sum_rows<T, W, SMALL>(a, dout, s[i], s[i + 1], c, sum);
#pragma unroll
            for (int j = 0; j < W; ++j) sum[j] *= a.scale;
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j) sum[j] = 0.0f;
        }
        Piece<T, W, SMALL>::template put<STREAM>(grad + (row0 + i) * a.D + c, a.D, sum);
    }
}

// A long row is joined by the threads of the piece that it begins in (it is the row of that piece's last position).
template <typename T, bool SMALL>
__global__ __launch_bounds__(256) void join_kernel(GradArgs a, T* __restrict__ grad) {
    constexpr int W = Wide<T>::V;
    const int64_t k = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t j = k / a.cpr;
    const int c = piece_start<W, SMALL>(static_cast<int>(k - j * a.cpr), a.D);
    const int64_t from = j * a.piece;
    const int total = a.start[a.V];
    if (from >= total) return;
    const int64_t to = from + a.piece < total ? from + a.piece : total;
    const int row = a.ids[a.order[to - 1]];
    const int s = a.start[row], e = a.start[row + 1];
    if (e - s <= a.piece || s < from) return;
    const int64_t last = (e - 1) / a.piece;
    float sum[W], v[W];
    Piece<float, W, SMALL> part;
    part.load(a.partial + (2 * j + (s > from)) * a.D + c, a.D);
    part.get(sum);
    constexpr int U = 8;
    for (int64_t q = j + 1; q <= last; q += U) {
        Piece<float, W, SMALL> more[U];
#pragma unroll
        for (int u = 0; u < U; ++u) more[u].load(a.partial + 2 * (q + u <= last ? q + u : last) * a.D + c, a.D);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            more[u].get(v);
#pragma unroll
            for (int i = 0; i < W; ++i) sum[i] += q + u <= last ? v[i] : 0.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < W; ++i) sum[i] *= a.scale;
    Piece<T, W, SMALL>::put(grad + static_cast<int64_t>(row) * a.D + c, a.D, sum);
}

// Sorted positions that a partial sum covers at most.  The sums of pieces run beside those of all other rows, those of their
// results after them: long pieces where there is much beside them (32768 positions, 100003 rows: join 5 us, with pieces of 32 10), short ones in
// small batches (2048 positions).
inline int piece_of(int64_t n) { return n >= 16384 ? 128 : 32; }
inline int64_t pieces_of(int64_t n) { return n > piece_of(n) ? (n + piece_of(n) - 1) / piece_of(n) : 0; }

// Rows whose ends lie inside a line of memory (128 bytes) are written past the caches in parts of lines; where few of them hold
// anything, the index clears all rows in one sweep of whole lines and the rows that hold something are written once more.  us, swept / row
// by row (results in turn in five places): 1653 positions into 93091 rows of 666 floats 59 / 77, 4096 into 98000 64 / 82, 2048 into 500000 of
// 100 bfloat16 36 / 58, 512 into 300000 of 33 floats 23 / 32; at eight rows a position 8192 into 65536 of 666 floats 53 / 59, 2048 into
// 16384 22.3 / 21.4; at three 32768 into 100000 of 301 floats 62 / 61.  Rows of whole lines: 2048 into 100003 of 512 floats 50 / 44.
inline bool rows_are_few(int64_t n, int V, int64_t row_bytes) { return V >= 8 * n && row_bytes % 128 != 0 && past_caches(V * row_bytes); }

template <typename T, bool SMALL>
hipError_t embed_of(const void* table, int V, int D, int64_t table_row, const int32_t* ids, int64_t n, float scale, void* out, hipStream_t st) {
    const int cpr = pieces_of_row(D, Wide<T>::V);
    // positions a workgroup: its threads' kItems pieces, one position at least
    const int per_block = cpr >= 256 * kItems ? 1 : 256 * kItems / cpr;
    if (!fits((n + per_block - 1) / per_block, 256)) return hipErrorInvalidValue;
    // (rows narrower than a piece go out element by element: through the caches)
    const auto kernel = past_caches(n * D * static_cast<int64_t>(sizeof(T))) ? embed_kernel<T, SMALL, !SMALL> : embed_kernel<T, SMALL, false>;
    kernel<<<static_cast<unsigned>((n + per_block - 1) / per_block), 256, 0, st>>>(static_cast<const T*>(table), V, D, table_row, ids, n, scale,
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
    const int cpr = pieces_of_row(D, Wide<T>::V);
    const GradArgs a{ids, order, start, n, N < 1 ? 1 : N, V, D, cpr, piece_of(n), scale, partial};
    const int64_t pieces = pieces_of(n);  // without a row that can be long there is nothing to cut
    const int64_t piece_blocks = (2 * pieces * cpr + 255) / 256;
    // Four rows a thread once that leaves a quarter of a million threads: their starts are loaded together, and rows of zeros cost little else.
    const bool four = static_cast<int64_t>(V) * cpr >= (int64_t{1} << 20);
    const bool sparse = rows_are_few(n, V, D * static_cast<int64_t>(sizeof(T)));
    const int64_t row_blocks = ((sparse ? n : four ? (V + 3) / 4 : V) * static_cast<int64_t>(cpr) + 255) / 256;
    if (!fits(piece_blocks + row_blocks, 256)) return hipErrorInvalidValue;
    const int bytes = static_cast<int>(sizeof(int32_t)) * kIndexWaves * (plan.range + kKept);
    static std::atomic<uint64_t> asked{0};
    if (const hipError_t e = ask_lds(reinterpret_cast<const void*>(index_kernel), static_cast<int>(sizeof(int32_t)) * kIndexWaves * (kMaxRange + kKept), asked); e != hipSuccess)
        return e;
    const int64_t table_bytes = static_cast<int64_t>(V) * D * static_cast<int64_t>(sizeof(T));
    const bool stream = past_caches(table_bytes);  // (such a table has four rows a thread: 2^20 pieces are at most 16 MB)
    index_kernel<<<sparse && plan.workgroups < 256 ? 256 : plan.workgroups, kIndexThreads, bytes, st>>>(ids, n, V, plan.range, order, start, sparse ? static_cast<char*>(grad) : nullptr, table_bytes);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const auto rows = sparse ? rows_kernel<T, SMALL, 0, false> : !four ? rows_kernel<T, SMALL, 1, false>
                      : stream ? rows_kernel<T, SMALL, 4, !SMALL> : rows_kernel<T, SMALL, 4, false>;
    if (piece_blocks + row_blocks) rows<<<static_cast<unsigned>(piece_blocks + row_blocks), 256, 0, st>>>(a, dout.as<T>(), static_cast<T*>(grad), static_cast<int>(piece_blocks));
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
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
    return up256((static_cast<size_t>(V) + 1) * 4) + up256(static_cast<size_t>(n) * 4) + up256(static_cast<size_t>(pieces_of(n)) * 2 * D * 4) + 256;
}

hipError_t launch_embed_grad(int dtype, AnyRows dout, const int32_t* ids, int B, int N, int V, int D, float scale, void* grad, void* ws, hipStream_t st) {
    const auto of = dtype ? (D < Wide<uint16_t>::V ? embed_grad_of<uint16_t, true> : embed_grad_of<uint16_t, false>)
                          : (D < Wide<float>::V ? embed_grad_of<float, true> : embed_grad_of<float, false>);
    return of(dout, ids, B, N, V, D, scale, grad, ws, st);
}

}  // namespace enc
}  // namespace lccrf
