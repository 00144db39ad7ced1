// Group norm with an activation, channels last, and its gradient.
//
// A value takes some ten operations forwards and twice that backwards, so traffic bounds all of it.  A thread has a piece of W channels of
// one group: 16 bytes, or less where a group has fewer channels.  A group whose width is no multiple of W has its last piece moved back
// to end with it: what it shares with the piece before is computed and written twice, the same, and counted once.
// Means and sums of squares are taken in two passes over values in registers and joined pairwise with their counts,
//     n = n1 + n2,  d = mean2 - mean1,  mean = mean1 + d n2 / n,  M = M1 + M2 + d^2 n1 n2 / n,
// always in the same order: no difference of large numbers, however far the mean is from 0.
#include "lccrf_layers.h"

namespace lccrf {
namespace enc {
namespace {

// ---- pieces ---------------------------------------------------------------------------------------------------

template <typename T, int W> using Part = Piece<T, W, W == 1>;

struct Place {
    int c, group, skip;  // first channel; its group; how many of the channels the piece before has too
    template <int W> static __device__ __forceinline__ Place of(int piece, int ppg, int C) {
        const int g = piece / ppg, want = (piece - g * ppg) * W, at = want <= C - W ? want : C - W;
        return {g * C + at, g, want - at};
    }
};

__device__ __forceinline__ float dsilu(float y) {
    const float s = sigmoid(y);
    return s * fmaf(y, 1.0f - s, 1.0f);
}

struct Moments { float n, mean, m2; };
__device__ __forceinline__ Moments join(const Moments& a, const Moments& b) {
    const float n = a.n + b.n, share = b.n / n, d = b.mean - a.mean;
    const Moments both{n, fmaf(d, share, a.mean), a.m2 + fmaf(d * d, a.n * share, b.m2)};
    return b.n == 0.0f ? a : a.n == 0.0f ? b : both;
}

template <typename T> __device__ __forceinline__ const T* line(const AnyRows& r, int64_t b, int64_t l) {
    return static_cast<const T*>(r.data) + b * r.batch + l * r.row;
}

template <int W> __device__ __forceinline__ void weights_of(const NormIn& in, int c, float (&w)[W], float (&bias)[W]) {
#pragma unroll
    for (int j = 0; j < W; ++j) {
        w[j] = in.weight ? in.weight[c + j] : 1.0f;
        bias[j] = in.bias ? in.bias[c + j] : 0.0f;
    }
}

// ---- every position by itself ---------------------------------------------------------------------------------
// A team of `team` lanes has a group of a position, R pieces a lane, all of it in registers.  A wave's teams have `groups` groups of so many
// positions; a workgroup keeps to its groups, so that the gradient's sums over positions stay in registers.
struct Alone {
    int ppg, team, groups, tiles;  // pieces a group, lanes a team, groups a wave, such tiles of groups in all
    int64_t blocks;                // workgroups a tile
};

__device__ __forceinline__ float team_sum(float v, int team) {
    for (int k = 1; k < team; k *= 2) v += __shfl_xor(v, k);
    return v;
}

template <typename T, int W, int R, bool GRAD>
__global__ __launch_bounds__(256) void alone_kernel(NormIn in, AnyRows dout, Alone p, const float* __restrict__ given, T* __restrict__ out, float* __restrict__ stats,
                                                    float* __restrict__ partial) {
    __shared__ float sums[GRAD ? 4 * 64 * 2 * W : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = lane % p.team, team = lane / p.team, rows = 64 / p.team / p.groups;  // positions a wave
    const int tile = blockIdx.x % p.tiles, g = tile * p.groups + team % p.groups, C = in.D / in.G;
    const int64_t block = blockIdx.x / p.tiles, total = static_cast<int64_t>(in.B) * in.N;
    const bool is = g < in.G;
    int c[R], skip[R];  // skip W: no piece
    float w[R][W], bias[R][W], dw[GRAD ? R : 1][W], db[GRAD ? R : 1][W];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int k = t + r * p.team;
        const Place at = Place::of<W>((is ? g : 0) * p.ppg + (k < p.ppg ? k : 0), p.ppg, C);
        c[r] = at.c;
        skip[r] = is && k < p.ppg ? at.skip : W;
        weights_of<W>(in, c[r], w[r], bias[r]);
#pragma unroll
        for (int j = 0; j < W; ++j)
            if (GRAD) dw[r][j] = db[r][j] = 0.0f;
    }
    const float count = 1.0f / C;
    for (int64_t base = (block * 4 + wave) * rows; base < total; base += p.blocks * 4 * rows) {
        const int64_t pos = base + team / p.groups;
        const bool there = pos < total;
        const unsigned at = there ? static_cast<unsigned>(pos) : 0u;
        const int b = at / static_cast<unsigned>(in.N), l = at - b * in.N;
        const bool inside = there && is && l < length_at(in.lengths, b, in.N);
        float x[R][W], dy[GRAD ? R : 1][W];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            Part<T, W> v, d;
            const bool read = inside && skip[r] < W;
            if (read) {
                v.load(line<T>(in.x, b, l) + c[r], W);
                if (GRAD) d.load(line<T>(dout, b, l) + c[r], W);
                v.get(x[r]);
                if (GRAD) d.get(dy[r]);
            } else {
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    x[r][j] = 0.0f;
                    if (GRAD) dy[r][j] = 0.0f;
                }
            }
        }
        const int64_t unit = (static_cast<int64_t>(b) * in.N + l) * in.G + g;
        float mean = 0.0f, rstd = 0.0f;
        if (GRAD && given) {
            if (inside) {
                mean = given[2 * unit];
                rstd = given[2 * unit + 1];
            }
        } else {
            float s = 0.0f, m2 = 0.0f;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < W; ++j) s += j >= skip[r] ? x[r][j] : 0.0f;
            mean = team_sum(s, p.team) * count;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const float d = x[r][j] - mean;
                    m2 += j >= skip[r] ? d * d : 0.0f;
                }
            rstd = __builtin_amdgcn_rsqf(fmaf(team_sum(m2, p.team), count, in.eps));
        }
        if constexpr (!GRAD) {
            if (stats && there && is && t == 0) {
                stats[2 * unit] = inside ? mean : 0.0f;
                stats[2 * unit + 1] = inside ? rstd : 0.0f;
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float o[W];
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const float y = fmaf((x[r][j] - mean) * rstd, w[r][j], bias[r][j]);
                    o[j] = inside ? in.silu ? silu(y) : y : 0.0f;
                }
                if (there && skip[r] < W) Part<T, W>::put(out + (static_cast<int64_t>(b) * in.N + l) * in.D + c[r], W, o);
            }
        } else {
            float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const float hat = (x[r][j] - mean) * rstd;
                    x[r][j] = hat;
                    if (in.silu) dy[r][j] *= dsilu(fmaf(hat, w[r][j], bias[r][j]));
                    const bool counts = inside && j >= skip[r];
                    dw[r][j] += counts ? dy[r][j] * hat : 0.0f;
                    db[r][j] += counts ? dy[r][j] : 0.0f;
                    dy[r][j] *= w[r][j];
                    s1 += counts ? dy[r][j] : 0.0f;
                    s2 += counts ? dy[r][j] * hat : 0.0f;
                }
            s1 = team_sum(s1, p.team) * count;
            s2 = team_sum(s2, p.team) * count;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float o[W];
#pragma unroll
                for (int j = 0; j < W; ++j) o[j] = inside ? rstd * (dy[r][j] - fmaf(x[r][j], s2, s1)) : 0.0f;
                if (there && skip[r] < W) Part<T, W>::put(out + (static_cast<int64_t>(b) * in.N + l) * in.D + c[r], W, o);
            }
        }
    }
    if constexpr (GRAD) {
        if (!partial) return;
        const int many = 64 / (p.team * p.groups);  // teams of a wave with the same group
#pragma unroll
        for (int r = 0; r < R; ++r) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < W; ++j) {
                sums[((wave * 2 + 0) * W + j) * 64 + lane] = dw[r][j];
                sums[((wave * 2 + 1) * W + j) * 64 + lane] = db[r][j];
            }
            __syncthreads();
            if (wave < 2 && team < p.groups) {  // wave 0: dweight, wave 1: dbias
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    float s = 0.0f;
                    for (int v = 0; v < 4; ++v)
                        for (int m = 0; m < many; ++m) s += sums[((v * 2 + wave) * W + j) * 64 + m * p.team * p.groups + lane];
                    if (j >= skip[r]) partial[(block * 2 + wave) * in.D + c[r] + j] = s;
                }
            }
        }
    }
}

// Groups too wide for a wave's registers: a workgroup has a group of a position and passes over it once for the mean, once for the squares, once to
// write (the caches hold it).
__device__ __forceinline__ float block_sum(float v, float* lds) {
    for (int k = 1; k < 64; k *= 2) v += __shfl_xor(v, k);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return lds[0] + lds[1] + lds[2] + lds[3];
}

template <typename T, int W, bool GRAD>
__global__ __launch_bounds__(256) void wide_kernel(NormIn in, AnyRows dout, int ppg, const float* __restrict__ given, T* __restrict__ out, float* __restrict__ stats) {
    __shared__ float lds[4];
    const int64_t total = static_cast<int64_t>(in.B) * in.N * in.G;
    const int C = in.D / in.G;
    for (int64_t unit = blockIdx.x; unit < total; unit += gridDim.x) {
        const int64_t pos = unit / in.G;
        const int g = static_cast<int>(unit - pos * in.G), b = static_cast<int>(pos / in.N), l = static_cast<int>(pos - static_cast<int64_t>(b) * in.N);
        T* o = out + pos * in.D;
        if (l >= length_at(in.lengths, b, in.N)) {
            const float zero[W] = {};
            for (int k = threadIdx.x; k < ppg; k += 256) Part<T, W>::put(o + Place::of<W>(g * ppg + k, ppg, C).c, W, zero);
            if (!GRAD && stats && threadIdx.x < 2) stats[2 * unit + threadIdx.x] = 0.0f;
            continue;
        }
        const T *px = line<T>(in.x, b, l), *pd = GRAD ? line<T>(dout, b, l) : nullptr;
        const auto sum = [&](auto of) {
            float s = 0.0f;
            for (int k = threadIdx.x; k < ppg; k += 256) {
                const Place at = Place::of<W>(g * ppg + k, ppg, C);
                Part<T, W> v;
                float x[W];
                v.load(px + at.c, W);
                v.get(x);
#pragma unroll
                for (int j = 0; j < W; ++j) s += j >= at.skip ? of(x[j]) : 0.0f;
            }
            return block_sum(s, lds) / C;
        };
        float mean, rstd;
        if (GRAD && given) {
            mean = given[2 * unit];
            rstd = given[2 * unit + 1];
        } else {
            mean = sum([](float x) { return x; });
            rstd = __builtin_amdgcn_rsqf(sum([=](float x) { return (x - mean) * (x - mean); }) + in.eps);
            if (stats && threadIdx.x == 0) {
                stats[2 * unit] = mean;
                stats[2 * unit + 1] = rstd;
            }
        }
        float s1 = 0.0f, s2 = 0.0f;
        for (int write = GRAD ? 0 : 1; write < 2; ++write) {
            for (int k = threadIdx.x; k < ppg; k += 256) {
                const Place at = Place::of<W>(g * ppg + k, ppg, C);
                Part<T, W> v, d;
                float x[W], w[W], bias[W], dy[W];
                v.load(px + at.c, W);
                if (GRAD) d.load(pd + at.c, W);
                weights_of<W>(in, at.c, w, bias);
                v.get(x);
                if (GRAD) d.get(dy);
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const float hat = (x[j] - mean) * rstd, y = fmaf(hat, w[j], bias[j]);
                    if (GRAD) {
                        const float dh = (in.silu ? dy[j] * dsilu(y) : dy[j]) * w[j];
                        if (!write && j >= at.skip) {
                            s1 += dh;
                            s2 += dh * hat;
                        }
                        x[j] = rstd * (dh - fmaf(hat, s2, s1));
                    } else {
                        x[j] = in.silu ? silu(y) : y;
                    }
                }
                if (write) Part<T, W>::put(o + at.c, W, x);
            }
            if (GRAD && !write) {
                s1 = block_sum(s1, lds) / C;
                s2 = block_sum(s2, lds) / C;
            }
        }
    }
}

// ---- whole sequences ------------------------------------------------------------------------------------------
// Workgroups are lx pieces wide and ly = 256 / lx positions high and go over a chunk of a sequence's positions.
struct Span {
    int ppg, pieces, lx, tiles;  // pieces a group and a row, across a workgroup, such tiles
    int chunk, chunks;           // positions a workgroup, workgroups a sequence
};
struct SpanPlace { int b, chunk, piece, ty, ly; };
__device__ __forceinline__ SpanPlace span_place(const Span& p) {
    const unsigned rest = blockIdx.x / p.tiles, tile = blockIdx.x - rest * p.tiles, b = rest / p.chunks;
    const int tx = threadIdx.x % p.lx;
    return {static_cast<int>(b), static_cast<int>(rest - b * p.chunks), static_cast<int>(tile) * p.lx + tx, static_cast<int>(threadIdx.x) / p.lx, 256 / p.lx};
}

// Moments of every piece over a chunk: [B][chunks][pieces][2] (mean, M; the count follows from the lengths).
constexpr int kBatch = 4;  // positions in flight
template <typename T, int W>
__global__ __launch_bounds__(256) void moments_kernel(NormIn in, Span p, float* __restrict__ made) {
    __shared__ Moments lds[256];
    const SpanPlace my = span_place(p);
    const int len = length_at(in.lengths, my.b, in.N), begin = my.chunk * p.chunk, stop = len - begin < p.chunk ? len : begin + p.chunk;
    if (begin >= len) return;  // nobody looks at these
    const bool is = my.piece < p.pieces;
    const Place at = Place::of<W>(is ? my.piece : 0, p.ppg, in.D / in.G);
    Moments m{0.0f, 0.0f, 0.0f};
    for (int l = begin + my.ty; l < stop; l += kBatch * my.ly) {
        Part<T, W> v[kBatch];
        float x[kBatch][W], s = 0.0f, q = 0.0f;
        int rows = 0;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const bool on = l + u * my.ly < stop;
            v[u].load(line<T>(in.x, my.b, on ? l + u * my.ly : l) + at.c, W);
            rows += on;
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            v[u].get(x[u]);
#pragma unroll
            for (int j = 0; j < W; ++j) s += u < rows && j >= at.skip ? x[u][j] : 0.0f;
        }
        const float n = static_cast<float>(rows * (W - at.skip)), mean = s / n;
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
#pragma unroll
            for (int j = 0; j < W; ++j) q += u < rows && j >= at.skip ? (x[u][j] - mean) * (x[u][j] - mean) : 0.0f;
        m = join(m, {n, mean, q});
    }
    lds[threadIdx.x] = m;
    for (int k = 128; k >= p.lx; k /= 2) {  // lx is a power of two
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < k) lds[threadIdx.x] = m = join(m, lds[threadIdx.x + k]);
    }
    if (my.ty == 0 && is) {
        float* to = made + ((static_cast<int64_t>(my.b) * p.chunks + my.chunk) * p.pieces + my.piece) * 2;
        to[0] = m.mean;
        to[1] = m.m2;
    }
}

// A workgroup joins a group's moments: stats [B][G][2].
template <int W>
__global__ __launch_bounds__(256) void stats_kernel(NormIn in, Span p, const float* __restrict__ made, float* __restrict__ stats) {
    __shared__ Moments lds[256];
    const int64_t unit = blockIdx.x, b = unit / in.G;
    const int g = static_cast<int>(unit - b * in.G), len = length_at(in.lengths, static_cast<int>(b), in.N);
    const int chunks = (len - 1) / p.chunk + 1, C = in.D / in.G;  // (len 0: all of one chunk of no positions)
    Moments m{0.0f, 0.0f, 0.0f};
    for (int64_t e = threadIdx.x; len > 0 && e < static_cast<int64_t>(chunks) * p.ppg; e += 256) {
        const int k = static_cast<int>(e / p.ppg), piece = static_cast<int>(e - static_cast<int64_t>(k) * p.ppg);
        const Place at = Place::of<W>(g * p.ppg + piece, p.ppg, C);
        const int rows = len - k * p.chunk < p.chunk ? len - k * p.chunk : p.chunk;
        const float* from = made + ((b * p.chunks + k) * p.pieces + g * p.ppg + piece) * 2;
        m = join(m, {static_cast<float>(rows) * (W - at.skip), from[0], from[1]});
    }
    lds[threadIdx.x] = m;
    for (int k = 128; k >= 1; k /= 2) {
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < k) lds[threadIdx.x] = m = join(m, lds[threadIdx.x + k]);
    }
    if (threadIdx.x == 0) {
        stats[2 * unit] = m.mean;
        stats[2 * unit + 1] = len > 0 ? __builtin_amdgcn_rsqf(m.m2 / m.n + in.eps) : 0.0f;
    }
}

// sums [B][G][2]: the means of dhat and of dhat hat (GRAD).
template <typename T, int W, bool GRAD>
__global__ __launch_bounds__(256) void apply_kernel(NormIn in, AnyRows dout, Span p, const float* __restrict__ stats, const float* __restrict__ sums, T* __restrict__ out) {
    const SpanPlace my = span_place(p);
    if (my.piece >= p.pieces) return;
    const int len = length_at(in.lengths, my.b, in.N), begin = my.chunk * p.chunk, stop = in.N - begin < p.chunk ? in.N : begin + p.chunk;
    const int end = len < begin ? begin : len < stop ? len : stop;
    const Place at = Place::of<W>(my.piece, p.ppg, in.D / in.G);
    T* o = out + static_cast<int64_t>(my.b) * in.N * in.D + at.c;
    const int64_t unit = static_cast<int64_t>(my.b) * in.G + at.group;
    float w[W], bias[W];
    weights_of<W>(in, at.c, w, bias);
    const float mean = stats[2 * unit], rstd = stats[2 * unit + 1], s1 = GRAD ? sums[2 * unit] : 0.0f, s2 = GRAD ? sums[2 * unit + 1] : 0.0f;
    int l = begin + my.ty;
    for (; l < end; l += kBatch * my.ly) {
        Part<T, W> v[kBatch], d[GRAD ? kBatch : 1];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int at_l = l + u * my.ly < end ? l + u * my.ly : l;
            v[u].load(line<T>(in.x, my.b, at_l) + at.c, W);
            if (GRAD) d[u].load(line<T>(dout, my.b, at_l) + at.c, W);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            float x[W], dy[W];
            v[u].get(x);
            if (GRAD) d[u].get(dy);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const float hat = (x[j] - mean) * rstd, y = fmaf(hat, w[j], bias[j]);
                if (GRAD) x[j] = rstd * ((in.silu ? dy[j] * dsilu(y) : dy[j]) * w[j] - fmaf(hat, s2, s1));
                else x[j] = in.silu ? silu(y) : y;
            }
            if (l + u * my.ly < end) Part<T, W>::put(o + static_cast<int64_t>(l + u * my.ly) * in.D, W, x);
        }
    }
    const float zero[W] = {};
    for (l = end + my.ty; l < stop; l += my.ly) Part<T, W>::put(o + static_cast<int64_t>(l) * in.D, W, zero);
}

// Sums of dy hat and dy over a chunk's positions: [B * chunks][2][D] (ALONE: every position has its own statistics, B is 1 and N all positions).
template <typename T, int W, bool ALONE>
__global__ __launch_bounds__(256) void columns_kernel(NormIn in, AnyRows dout, Span p, const float* __restrict__ stats, float* __restrict__ partial) {
    __shared__ float lds[256 * 2 * W];
    const SpanPlace my = span_place(p);
    const int all = ALONE ? in.B * in.N : in.N;
    const int len = ALONE ? all : length_at(in.lengths, my.b, in.N), begin = my.chunk * p.chunk;
    const int stop = len - begin < p.chunk ? len : begin + p.chunk;
    const bool is = my.piece < p.pieces;
    const Place at = Place::of<W>(is ? my.piece : 0, p.ppg, in.D / in.G);
    float w[W], bias[W], dw[W] = {}, db[W] = {};
    weights_of<W>(in, at.c, w, bias);
    const int64_t unit = static_cast<int64_t>(my.b) * in.G + at.group;
    float mean = 0.0f, rstd = 0.0f;
    if (!ALONE) {
        mean = stats[2 * unit];
        rstd = stats[2 * unit + 1];
    }
    for (int l = begin + my.ty; l < stop; l += kBatch * my.ly) {
        Part<T, W> v[kBatch], d[kBatch];
        float means[kBatch], rstds[kBatch];
        bool on[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            on[u] = l + u * my.ly < stop;
            const int pos = on[u] ? l + u * my.ly : l, b = ALONE ? pos / in.N : my.b, row = ALONE ? pos - b * in.N : pos;
            if (ALONE) {
                on[u] = on[u] && row < length_at(in.lengths, b, in.N);
                means[u] = stats[(static_cast<int64_t>(pos) * in.G + at.group) * 2];
                rstds[u] = stats[(static_cast<int64_t>(pos) * in.G + at.group) * 2 + 1];
            }
            if (!ALONE || on[u]) {
                v[u].load(line<T>(in.x, b, row) + at.c, W);
                d[u].load(line<T>(dout, b, row) + at.c, W);
            }
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            float x[W], dy[W];
            v[u].get(x);
            d[u].get(dy);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const float hat = (x[j] - (ALONE ? means[u] : mean)) * (ALONE ? rstds[u] : rstd);
                const float g = in.silu ? dy[j] * dsilu(fmaf(hat, w[j], bias[j])) : dy[j];
                dw[j] += on[u] ? g * hat : 0.0f;
                db[j] += on[u] ? g : 0.0f;
            }
        }
    }
#pragma unroll
    for (int j = 0; j < W; ++j) {
        lds[(2 * j) * 256 + threadIdx.x] = dw[j];
        lds[(2 * j + 1) * 256 + threadIdx.x] = db[j];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * W * p.lx; e += 256) {
        const int x = e % p.lx, k = e / p.lx, piece = my.piece - static_cast<int>(threadIdx.x) % p.lx + x;
        if (piece >= p.pieces) continue;
        const Place to = Place::of<W>(piece, p.ppg, in.D / in.G);
        float s = 0.0f;
        for (int y = 0; y < my.ly; ++y) s += lds[k * 256 + y * p.lx + x];
        if (k / 2 >= to.skip) partial[((static_cast<int64_t>(my.b) * p.chunks + my.chunk) * 2 + k % 2) * in.D + to.c + k / 2] = s;
    }
}

// A workgroup joins a group's sums: [B][G][2], the means of dhat and dhat hat.
__global__ __launch_bounds__(256) void group_sums_kernel(NormIn in, int chunks, const float* __restrict__ partial, float* __restrict__ sums) {
    __shared__ float lds[4];
    const int64_t unit = blockIdx.x, b = unit / in.G;
    const int g = static_cast<int>(unit - b * in.G), len = length_at(in.lengths, static_cast<int>(b), in.N), C = in.D / in.G;
    float s1 = 0.0f, s2 = 0.0f;
    for (int64_t e = threadIdx.x; e < static_cast<int64_t>(chunks) * C; e += 256) {
        const int64_t k = e / C;
        const int c = g * C + static_cast<int>(e - k * C);
        const float w = in.weight ? in.weight[c] : 1.0f, *from = partial + (b * chunks + k) * 2 * in.D + c;
        s2 = fmaf(w, from[0], s2);
        s1 = fmaf(w, from[in.D], s1);
    }
    s1 = block_sum(s1, lds);
    s2 = block_sum(s2, lds);
    if (threadIdx.x == 0) {
        const float n = static_cast<float>(len) * C;
        sums[2 * unit] = len > 0 ? s1 / n : 0.0f;
        sums[2 * unit + 1] = len > 0 ? s2 / n : 0.0f;
    }
}

// dweight and dbias from [parts][2][D]: workgroups of 64 channels, sixteen threads a channel.
__global__ __launch_bounds__(1024) void channel_sums_kernel(const float* __restrict__ partial, int64_t parts, int D, float* __restrict__ dweight, float* __restrict__ dbias) {
    __shared__ float lds[16][64];
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6, k = blockIdx.y, ch = blockIdx.x * 64 + x;
    float* to = k ? dbias : dweight;
    if (!to) return;
    float s = 0.0f;
    if (ch < D)
        for (int64_t q = y; q < parts; q += 16) s += partial[(q * 2 + k) * D + ch];
    lds[y][x] = s;
    __syncthreads();
    if (y || ch >= D) return;
    for (int i = 1; i < 16; ++i) s += lds[i][x];
    to[ch] = s;
}

// ---- launches -------------------------------------------------------------------------------------------------

int piece_width(int dtype, int C) {
    int w = dtype ? 8 : 4;
    while (w > C) w /= 2;
    return w;
}

constexpr int kMostPieces = 4;  // a lane's, in registers

bool alone_fits(int ppg) { return ppg <= 64 * kMostPieces; }
// Lanes a team and pieces a lane: one each as long as a wave has the lanes; 3 pieces where that leaves fewer of them without one.
void team_of(int ppg, int& team, int& pieces) {
    team = 1;
    while (team < 64 && team < ppg) team *= 2;
    pieces = (ppg + team - 1) / team;
    if (pieces == 1 && team >= 4 && 3 * (team / 4) >= ppg) {
        team /= 4;
        pieces = 3;
    }
}

Alone alone_plan(int dtype, int B, int N, int D, int G, int& pieces) {
    Alone p;
    const int C = D / G, W = piece_width(dtype, C);
    p.ppg = (C - 1) / W + 1;
    team_of(p.ppg, p.team, pieces);
    p.groups = 1;
    while (p.groups < 64 / p.team && p.groups < G) p.groups *= 2;
    p.tiles = (G - 1) / p.groups + 1;
    const int64_t rows = 4 * (64 / p.team / p.groups), all = (static_cast<int64_t>(B) * N + rows - 1) / rows;
    int64_t most = 2048 / p.tiles;
    if (most < 1) most = 1;
    p.blocks = all < most ? all : most;
    return p;
}

Span span_plan(int dtype, int B, int N, int D, int G) {
    Span p;
    const int C = D / G, W = piece_width(dtype, C);
    p.ppg = (C - 1) / W + 1;
    p.pieces = p.ppg * G;
    p.lx = 1;
    while (p.lx < 64 && p.lx < p.pieces) p.lx *= 2;
    p.tiles = (p.pieces - 1) / p.lx + 1;
    const int least = kBatch * (256 / p.lx);  // a chunk's positions: as many as keep 1024 workgroups, at most 16 batches of a thread
    p.chunk = 16 * least;
    while (p.chunk > least && static_cast<int64_t>(B) * p.tiles * ((N - 1) / p.chunk + 1) < 1024) p.chunk /= 2;
    p.chunks = (N - 1) / p.chunk + 1;
    return p;
}

size_t moments_bytes(const Span& p, int B) { return up256(static_cast<size_t>(B) * p.chunks * p.pieces * 8); }
size_t stats_bytes(int64_t units) { return up256(static_cast<size_t>(units) * 8); }
size_t partial_bytes(int64_t parts, int D) { return up256(static_cast<size_t>(parts) * 2 * D * 4); }

template <typename T, int W, bool GRAD>
hipError_t alone_of(const NormIn& in, AnyRows dout, const Alone& p, int pieces, const float* given, void* out, float* stats, float* partial, hipStream_t st) {
    if (!fits(p.blocks * p.tiles, 256)) return hipErrorInvalidValue;
    auto kernel = alone_kernel<T, W, 1, GRAD>;
    if constexpr (W == Wide<T>::V) {  // narrower pieces are at most two a group
        kernel = pieces <= 1 ? kernel : pieces == 2 ? alone_kernel<T, W, 2, GRAD> : pieces == 3 ? alone_kernel<T, W, 3, GRAD> : alone_kernel<T, W, 4, GRAD>;
    }
    kernel<<<static_cast<unsigned>(p.blocks * p.tiles), 256, 0, st>>>(in, dout, p, given, static_cast<T*>(out), stats, partial);
    return hipGetLastError();
}

constexpr int64_t kWideBlocks = 1 << 16;

struct Outs {
    void* out;  // or dx
    float *stats, *dweight, *dbias;
};

template <typename T, int W>
hipError_t norm_of(int dtype, const NormIn& in, const Outs& o, void* ws, hipStream_t st) {
    if (in.alone) {
        int pieces;
        const Alone p = alone_plan(dtype, in.B, in.N, in.D, in.G, pieces);
        if (alone_fits(p.ppg)) return alone_of<T, W, false>(in, {}, p, pieces, nullptr, o.out, o.stats, nullptr, st);
        if constexpr (W == Wide<T>::V) {
            const int64_t units = static_cast<int64_t>(in.B) * in.N * in.G;
            wide_kernel<T, W, false><<<static_cast<unsigned>(units < kWideBlocks ? units : kWideBlocks), 256, 0, st>>>(in, {}, p.ppg, nullptr, static_cast<T*>(o.out), o.stats);
        }
        return hipGetLastError();
    }
    const Span p = span_plan(dtype, in.B, in.N, in.D, in.G);
    const int64_t blocks = static_cast<int64_t>(in.B) * p.chunks * p.tiles;
    if (!fits(blocks, 256) || !fits(static_cast<int64_t>(in.B) * in.G, 256)) return hipErrorInvalidValue;
    float* made = static_cast<float*>(ws);
    float* stats = o.stats ? o.stats : reinterpret_cast<float*>(static_cast<char*>(ws) + moments_bytes(p, in.B));
    moments_kernel<T, W><<<static_cast<unsigned>(blocks), 256, 0, st>>>(in, p, made);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    stats_kernel<W><<<static_cast<unsigned>(in.B * in.G), 256, 0, st>>>(in, p, made, stats);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || !o.out) return e;
    apply_kernel<T, W, false><<<static_cast<unsigned>(blocks), 256, 0, st>>>(in, {}, p, stats, nullptr, static_cast<T*>(o.out));
    return hipGetLastError();
}

hipError_t channel_sums(const float* partial, int64_t parts, const NormIn& in, const Outs& o, hipStream_t st) {
    channel_sums_kernel<<<dim3(pieces_of_row(in.D, 64), 2), 1024, 0, st>>>(partial, parts, in.D, o.dweight, o.dbias);
    return hipGetLastError();
}

template <typename T, int W>
hipError_t norm_grad_of(int dtype, AnyRows dout, const NormIn& in, const float* stats, const Outs& o, void* ws, hipStream_t st) {
    char* room = static_cast<char*>(ws);
    const bool sums = o.dweight || o.dbias;
    if (in.alone) {
        int pieces;
        const Alone p = alone_plan(dtype, in.B, in.N, in.D, in.G, pieces);
        float* partial = reinterpret_cast<float*>(room);
        if (alone_fits(p.ppg)) {
            if (const hipError_t e = alone_of<T, W, true>(in, dout, p, pieces, stats, o.out, nullptr, sums ? partial : nullptr, st); e != hipSuccess || !sums) return e;
            return channel_sums(partial, p.blocks, in, o, st);
        }
        if constexpr (W == Wide<T>::V) {
            const int64_t units = static_cast<int64_t>(in.B) * in.N * in.G;
            const Span q = span_plan(dtype, 1, in.B * in.N, in.D, in.G);
            if (!fits(static_cast<int64_t>(q.chunks) * q.tiles, 256)) return hipErrorInvalidValue;
            float* made = reinterpret_cast<float*>(room + partial_bytes(q.chunks, in.D));
            wide_kernel<T, W, true><<<static_cast<unsigned>(units < kWideBlocks ? units : kWideBlocks), 256, 0, st>>>(in, dout, p.ppg, stats, static_cast<T*>(o.out), stats ? nullptr : made);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess || !sums) return e;
            columns_kernel<T, W, true><<<static_cast<unsigned>(q.chunks * q.tiles), 256, 0, st>>>(in, dout, q, stats ? stats : made, partial);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
            return channel_sums(partial, q.chunks, in, o, st);
        }
        return hipErrorInvalidValue;
    }
    const Span p = span_plan(dtype, in.B, in.N, in.D, in.G);
    const int64_t blocks = static_cast<int64_t>(in.B) * p.chunks * p.tiles, units = static_cast<int64_t>(in.B) * in.G;
    if (!fits(blocks, 256) || !fits(units, 256)) return hipErrorInvalidValue;
    float* partial = reinterpret_cast<float*>(room);
    room += partial_bytes(static_cast<int64_t>(in.B) * p.chunks, in.D);
    float* means = reinterpret_cast<float*>(room);
    room += stats_bytes(units);
    if (!stats) {
        float* made = reinterpret_cast<float*>(room);
        if (const hipError_t e = norm_of<T, W>(dtype, in, {nullptr, made, nullptr, nullptr}, room + stats_bytes(units), st); e != hipSuccess) return e;
        stats = made;
    }
    columns_kernel<T, W, false><<<static_cast<unsigned>(blocks), 256, 0, st>>>(in, dout, p, stats, partial);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    group_sums_kernel<<<static_cast<unsigned>(units), 256, 0, st>>>(in, p.chunks, partial, means);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    apply_kernel<T, W, true><<<static_cast<unsigned>(blocks), 256, 0, st>>>(in, dout, p, stats, means, static_cast<T*>(o.out));
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || !sums) return e;
    return channel_sums(partial, static_cast<int64_t>(in.B) * p.chunks, in, o, st);
}

#define LCCRF_BY_WIDTH(call)                      \
    switch (piece_width(dtype, in.D / in.G)) {    \
        case 8: return call(uint16_t, 8);         \
        case 4: return dtype ? call(uint16_t, 4) : call(float, 4); \
        case 2: return dtype ? call(uint16_t, 2) : call(float, 2); \
        default: return dtype ? call(uint16_t, 1) : call(float, 1); \
    }

}  // namespace

size_t norm_workspace(int dtype, int B, int N, int D, int G, bool alone) {
    if (alone) return 256;
    return moments_bytes(span_plan(dtype, B, N, D, G), B) + stats_bytes(static_cast<int64_t>(B) * G);
}

size_t norm_grad_workspace(int dtype, int B, int N, int D, int G, bool alone) {
    if (alone) {
        int pieces;
        const Alone p = alone_plan(dtype, B, N, D, G, pieces);
        if (alone_fits(p.ppg)) return partial_bytes(p.blocks, D);
        return partial_bytes(span_plan(dtype, 1, B * N, D, G).chunks, D) + stats_bytes(static_cast<int64_t>(B) * N * G);
    }
    const Span p = span_plan(dtype, B, N, D, G);
    const int64_t units = static_cast<int64_t>(B) * G;
    return partial_bytes(static_cast<int64_t>(B) * p.chunks, D) + 2 * stats_bytes(units) + norm_workspace(dtype, B, N, D, G, false);
}

hipError_t launch_norm(int dtype, const NormIn& in, void* out, float* stats, void* ws, hipStream_t st) {
    const Outs o{out, stats, nullptr, nullptr};
#define LCCRF_CALL(T, W) norm_of<T, W>(dtype, in, o, ws, st)
    LCCRF_BY_WIDTH(LCCRF_CALL)
#undef LCCRF_CALL
}

hipError_t launch_norm_grad(int dtype, AnyRows dout, const NormIn& in, const float* stats, void* dx, float* dweight, float* dbias, void* ws, hipStream_t st) {
    const Outs o{dx, nullptr, dweight, dbias};
#define LCCRF_CALL(T, W) norm_grad_of<T, W>(dtype, dout, in, stats, o, ws, st)
    LCCRF_BY_WIDTH(LCCRF_CALL)
#undef LCCRF_CALL
}

}  // namespace enc
}  // namespace lccrf
