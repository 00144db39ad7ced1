// Group norm with an activation, channels last, and its gradient.
//
// A value takes some ten operations forwards and twice that backwards, so traffic bounds all of it.  A thread has a piece of W channels of
// one group: 16 bytes, or less where a group has fewer channels.  A group whose width is no multiple of W has its last piece moved back
// to end with it: what it shares with the piece before is computed and written twice, the same, and counted once.
// Means and sums of squares are taken in two passes over values in registers and joined pairwise with their counts,
//     n = n1 + n2,  d = mean2 - mean1,  mean = mean1 + d n2 / n,  M = M1 + M2 + d^2 n1 n2 / n,
// always in the same order: no difference of large numbers, however far the mean is from 0.
#include "lccrf_ahead.h"
#include "lccrf_layers.h"

namespace lccrf {
namespace enc {
namespace {

// ---- pieces ---------------------------------------------------------------------------------------------------

// (again: of registers that hold the piece for several passes, widened in each where it is used and not kept so.)
template <typename T, int W> struct Part : Piece<T, W, W == 1> {
    __device__ __forceinline__ void again(float (&o)[W]) {
        if constexpr (W > 1) {
#pragma unroll
            for (int i = 0; i < static_cast<int>(W * sizeof(T) / 4); ++i) {
                uint32_t v = this->raw[i];
                asm volatile("" : "+v"(v));
                this->raw[i] = v;
            }
        }
        this->get(o);
    }
};

struct Place {
    int c, group, skip;  // first channel; its group; how many of the channels the piece before has too
    template <int W> static __device__ __forceinline__ Place of(int piece, int ppg, int C) {
        const int g = piece / ppg, want = (piece - g * ppg) * W, at = want <= C - W ? want : C - W;
        return {g * C + at, g, want - at};
    }
};

__device__ __forceinline__ float dsilu(float y) {
    const float s = sigmoid(y);
    return fmaf(s, fmaf(-y, s, y), s);  // s (1 + y (1 - s))
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
// positions; a workgroup keeps to its groups, so that the gradient's sums over positions stay in registers.  Forwards 64 x 512 x 1024 in 16 groups, bfloat16, 34 us
// (3.9 TB/s); with its gradient 128 x 128 x 1024 in eight, float, 77 us (3.5 TB/s), in seven of 1001, ragged, 89 - 93 (rows begin anywhere in a line).
struct Alone {
    int ppg, team, groups, tiles;  // pieces a group, lanes a team, groups a wave, such tiles of groups in all
    int64_t blocks;                // workgroups a tile
};

// EXACT: every lane has R pieces of its own, no channel twice.  ALL: the whole workgroup is one team.
template <typename T, int W, int R, bool GRAD, bool EXACT, bool ALL>
__global__ __launch_bounds__(256) void alone_kernel(NormIn in, AnyRows dout, Alone p, const float* __restrict__ given, T* __restrict__ out, float* __restrict__ stats,
                                                    float* __restrict__ partial) {
    __shared__ float sums[GRAD && !ALL ? 4 * 64 * 2 * W : 16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = ALL ? threadIdx.x : lane % p.team, team = ALL ? 0 : lane / p.team, rows = ALL ? 1 : 64 / p.team / p.groups;  // positions a wave
    const int tile = blockIdx.x % p.tiles, g = tile * p.groups + (ALL ? 0 : team % p.groups), C = in.D / in.G;
    const int64_t block = blockIdx.x / p.tiles, total = static_cast<int64_t>(in.B) * in.N;
    const int at_once = ALL ? 1 : 4 * rows;  // positions a workgroup
    // over the team; `which` of a position's four sums
    const auto team_sum = [&](float v, int which) {
        if (!ALL) return sum_across(v, p.team);
        v = sum_across(v, 64);
        if (lane == 0) sums[which * 4 + wave] = v;
        lds_sync();  // (a place is written again behind the wait of another such sum: all have read it)
        return sums[which * 4] + sums[which * 4 + 1] + sums[which * 4 + 2] + sums[which * 4 + 3];
    };
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
    // While a position is worked on the next one's values are on their way.  The length of the one after that is clamped, and so waited for, where it is loaded; the
    // position's own statistics, where given, come behind the next one's values and are waited for with them.
    struct Position {
        int b, l, len;
        bool there;
    };
    const int64_t high = p.blocks * at_once, first = ALL ? block : (block * 4 + wave) * rows + team / p.groups;
    const auto position = [&](int64_t pos) {
        Position q;
        q.there = pos < total;
        const unsigned at = q.there ? static_cast<unsigned>(pos) : 0u;
        q.b = at / static_cast<unsigned>(in.N);
        q.l = at - q.b * in.N;
        q.len = length_at(in.lengths, q.b, in.N);
        return q;
    };
    Part<T, W> v[R], d[GRAD ? R : 1];
    const auto fetch = [&](const Position& q) {
        if (q.there && is && q.l < q.len) {
            const T *px = line<T>(in.x, q.b, q.l), *pd = GRAD ? line<T>(dout, q.b, q.l) : nullptr;
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (EXACT || skip[r] < W) {
                    v[r].load(px + c[r], W);
                    if (GRAD) d[r].load(pd + c[r], W);
                }
        }
    };
    Position now = position(first), next = position(first + high);
    fetch(now);
    for (int64_t pos = first; pos - (ALL ? 0 : team / p.groups) < total; pos += high) {
        const Position after = position(pos + 2 * high);
        const int b = now.b, l = now.l;
        const bool there = now.there, inside = there && is && l < now.len;
        float x[R][W], dy[GRAD ? R : 1][W];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            v[r].get(x[r]);
            if (GRAD) d[r].get(dy[r]);
        }
        fetch(next);
        now = next;
        next = after;
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
                for (int j = 0; j < W; ++j) s += EXACT || j >= skip[r] ? x[r][j] : 0.0f;
            mean = team_sum(s, 0) * count;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const float away = x[r][j] - mean;
                    m2 = EXACT || j >= skip[r] ? fmaf(away, away, m2) : m2;
                }
            rstd = __builtin_amdgcn_rsqf(fmaf(team_sum(m2, 1), count, in.eps));
        }
        T* to = out + (static_cast<int64_t>(b) * in.N + l) * in.D;
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
                    const float y = fmaf(x[r][j] - mean, rstd * w[r][j], bias[r][j]);
                    o[j] = in.silu ? silu(y) : y;
                }
                if (!inside) {
#pragma unroll
                    for (int j = 0; j < W; ++j) o[j] = 0.0f;
                }
                if (there && is && (EXACT || skip[r] < W)) Part<T, W>::put(to + c[r], W, o);
            }
        } else {
            float s1 = 0.0f, s2 = 0.0f;
            if (inside) {  // (a team's lanes together)
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int j = 0; j < W; ++j) {
                        const float hat = (x[r][j] - mean) * rstd;
                        x[r][j] = hat;
                        if (in.silu) dy[r][j] *= dsilu(fmaf(hat, w[r][j], bias[r][j]));
                        if (EXACT || j >= skip[r]) {
                            dw[r][j] = fmaf(dy[r][j], hat, dw[r][j]);
                            db[r][j] += dy[r][j];
                        }
                        dy[r][j] *= w[r][j];
                        if (EXACT || j >= skip[r]) {
                            s1 += dy[r][j];
                            s2 = fmaf(dy[r][j], hat, s2);
                        }
                    }
            }
            s1 = team_sum(s1, 2) * count;
            s2 = team_sum(s2, 3) * count;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float o[W];
#pragma unroll
                for (int j = 0; j < W; ++j) o[j] = rstd * (dy[r][j] - fmaf(x[r][j], s2, s1));
                if (!inside) {
#pragma unroll
                    for (int j = 0; j < W; ++j) o[j] = 0.0f;
                }
                if (there && is && (EXACT || skip[r] < W)) Part<T, W>::put(to + c[r], W, o);
            }
        }
    }
    if constexpr (GRAD) {
        if (!partial) return;
        if constexpr (ALL) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < W; ++j)
                    if (j >= skip[r]) {
                        partial[block * 2 * in.D + c[r] + j] = dw[r][j];
                        partial[(block * 2 + 1) * in.D + c[r] + j] = db[r][j];
                    }
            return;
        }
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

// ---- whole sequences in registers ------------------------------------------------------------------------------
// Where a sequence's groups fit a workgroup's registers, they are read once: a workgroup has whole groups, `lx` pieces (a power of two) wide, of all positions, R
// pieces a thread.  `run` tiles side by side go to one XCD, one after another: where a tile is half a cache line wide the line is then fetched from memory once, and
// neighbouring lines of a row soon after each other.
struct Held {
    int ppg, lx, groups, tiles, threads, pieces, run;  // pieces a group; across a workgroup; groups a workgroup, such tiles; its threads, pieces each
};

// The sum of v over a group's pieces and all positions, for every thread of the group: first over the workgroup's positions, then over the pieces.
// lds: a float a thread, and lx.
__device__ __forceinline__ float held_sum(float v, const Held& p, float* lds, int tx, int group) {
    for (int k = p.lx; k < 64; k *= 2) v += __shfl_xor(v, k);
    const int wide = p.lx < 64 ? p.lx : 64, lane = threadIdx.x & 63, entries = (blockDim.x >> 6) * wide;
    __syncthreads();
    if (lane < wide) lds[(threadIdx.x >> 6) * wide + lane] = v;
    __syncthreads();
    float* columns = lds + blockDim.x;
    if (static_cast<int>(threadIdx.x) < p.lx) {
        float s = 0.0f;
        for (int e = threadIdx.x; e < entries; e += p.lx) s += lds[e];
        columns[threadIdx.x] = s;
    }
    __syncthreads();
    float s = 0.0f;
    if (group < p.groups)
        for (int k = 0; k < p.ppg; ++k) s += columns[group * p.ppg + k];
    return s;
}

template <typename T, int W, int R, bool GRAD>
__global__ __launch_bounds__(R > 4 ? 512 : 1024) void held_kernel(NormIn in, AnyRows dout, Held p, const float* __restrict__ given, T* __restrict__ out, float* __restrict__ stats,
                                                                  float* __restrict__ partial) {
    extern __shared__ float lds[];  // held_sum's; GRAD: [threads][W]
    const int tx = threadIdx.x & (p.lx - 1), ty = threadIdx.x / p.lx, ly = blockDim.x / p.lx, C = in.D / in.G;
    const unsigned run = p.run, rest = blockIdx.x / 8, work = (rest / run * 8 + blockIdx.x % 8) * run + rest % run;
    if (work >= static_cast<unsigned>(in.B) * p.tiles) return;
    const int b = work / p.tiles, tile = work - b * p.tiles, group = tx / p.ppg, g = tile * p.groups + group;
    const bool is = group < p.groups && g < in.G;
    const Place at = Place::of<W>(is ? g * p.ppg + tx - group * p.ppg : 0, p.ppg, C);
    const int len = length_at(in.lengths, b, in.N);
    const bool exact = at.skip == 0;
    Part<T, W> raw[R], draw[GRAD ? R : 1];
    {
        const T* px = line<T>(in.x, b, 0) + at.c;
        const T* pd = GRAD ? line<T>(dout, b, 0) + at.c : nullptr;
        const int64_t x_step = ly * in.x.row, d_step = ly * dout.row;
        px += ty * in.x.row;
        if (GRAD) pd += ty * dout.row;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r * ly >= len) break;
            if (is && ty + r * ly < len) {
                raw[r].load(px, W);
                if (GRAD) draw[r].load(pd, W);
            }
            px += x_step;
            pd += d_step;
        }
    }
    const float share = 1.0f / (static_cast<float>(len) * C);  // (len 0: nothing looks at it)
    const int64_t unit = static_cast<int64_t>(b) * in.G + g;
    float mean, rstd;
    if (GRAD && given) {
        mean = is ? given[2 * unit] : 0.0f;
        rstd = is ? given[2 * unit + 1] : 0.0f;
    } else {
        float s = 0.0f, q = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r * ly >= len) break;
            float x[W];
            raw[r].again(x);
            if (is && ty + r * ly < len) {
#pragma unroll
                for (int j = 0; j < W; ++j) s += exact || j >= at.skip ? x[j] : 0.0f;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        mean = held_sum(s, p, lds, tx, group) * share;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r * ly >= len) break;
            float x[W];
            raw[r].again(x);
            if (is && ty + r * ly < len) {
#pragma unroll
                for (int j = 0; j < W; ++j) q = exact || j >= at.skip ? fmaf(x[j] - mean, x[j] - mean, q) : q;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        rstd = __builtin_amdgcn_rsqf(fmaf(held_sum(q, p, lds, tx, group), share, in.eps));
        if (!GRAD && stats && is && ty == 0 && tx == group * p.ppg) {
            stats[2 * unit] = len > 0 ? mean : 0.0f;
            stats[2 * unit + 1] = len > 0 ? rstd : 0.0f;
        }
    }
    T* o = out + (static_cast<int64_t>(b) * in.N + ty) * in.D + at.c;
    const int64_t o_step = static_cast<int64_t>(ly) * in.D;
    float w[W], bias[W];
    int c = at.c;
    asm volatile("" : "+v"(c));  // fetched here and not in front of the sums, where they would take registers that hold values
    weights_of<W>(in, c, w, bias);
    const float zero[W] = {};
    if constexpr (!GRAD) {
        if (!is) return;
#pragma unroll
        for (int j = 0; j < W; ++j) w[j] *= rstd;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r * ly >= in.N) break;
            const int l = ty + r * ly;
            float x[W];
            raw[r].again(x);
            if (l < len) {
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const float y = fmaf(x[j] - mean, w[j], bias[j]);
                    x[j] = in.silu ? silu(y) : y;
                }
                Part<T, W>::put(o, W, x);
            } else if (l < in.N) {
                Part<T, W>::put(o, W, zero);
            }
            o += o_step;
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {
        float sums[2][W] = {};  // of dy hat, of dy
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r * ly >= len) break;
            float x[W], dy[W];
            raw[r].again(x);
            draw[r].again(dy);
            if (is && ty + r * ly < len) {
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const float hat = (x[j] - mean) * rstd, d = in.silu ? dy[j] * dsilu(fmaf(hat, w[j], bias[j])) : dy[j];
                    sums[0][j] = fmaf(d, hat, sums[0][j]);
                    sums[1][j] += d;
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        // over the positions, channel by channel; the first lx threads have them, write them and weigh them for the group
        const int wide = p.lx < 64 ? p.lx : 64, lane = threadIdx.x & 63, entries = (blockDim.x >> 6) * wide;
        float of_group[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int j = 0; j < W; ++j)
                for (int d = p.lx; d < 64; d *= 2) sums[k][j] += __shfl_xor(sums[k][j], d);
            __syncthreads();
            if (lane < wide) {
#pragma unroll
                for (int j = 0; j < W; ++j) lds[j * entries + (threadIdx.x >> 6) * wide + lane] = sums[k][j];
            }
            __syncthreads();
            if (static_cast<int>(threadIdx.x) < p.lx) {
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    float s = 0.0f;
                    for (int e = threadIdx.x; e < entries; e += p.lx) s += lds[j * entries + e];
                    of_group[k] += j >= at.skip ? w[j] * s : 0.0f;
                    if (partial && is && j >= at.skip) partial[(static_cast<int64_t>(b) * 2 + k) * in.D + at.c + j] = s;
                }
            }
        }
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < p.lx) {
            lds[threadIdx.x] = of_group[0];
            lds[p.lx + threadIdx.x] = of_group[1];
        }
        __syncthreads();
        if (!is) return;
        float s1 = 0.0f, s2 = 0.0f;
        for (int k = 0; k < p.ppg; ++k) {
            s2 += lds[group * p.ppg + k];
            s1 += lds[p.lx + group * p.ppg + k];
        }
        s1 *= -share * rstd;
        s2 *= -share * rstd;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r * ly >= in.N) break;
            const int l = ty + r * ly;
            float x[W], dy[W];
            raw[r].again(x);
            draw[r].again(dy);
            if (l < len) {
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const float hat = (x[j] - mean) * rstd, d = in.silu ? dy[j] * dsilu(fmaf(hat, w[j], bias[j])) : dy[j];
                    x[j] = fmaf(d, rstd * w[j], fmaf(hat, s2, s1));
                }
                Part<T, W>::put(o, W, x);
            } else if (l < in.N) {
                Part<T, W>::put(o, W, zero);
            }
            o += o_step;
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// ---- whole sequences ------------------------------------------------------------------------------------------
// Two passes: sums of every chunk of positions, then the results; the second finds most of what it reads in the memory-side cache.  Workgroups are lx pieces wide
// (whole groups, or one of the `parts` of a group that is wider), ly = 256 / lx positions high and go over a chunk of a sequence's positions.  What a group's
// chunks come to is joined by every workgroup of the second pass for its own groups, all in the same order: no launch between the two.  4 x 16384 x 512 in eight
// groups, bfloat16, lengths from 9000 on: 9 us and 22, of which 23 are the bytes' at the rate of a copy.
struct Span {
    int ppg, lx, groups, parts, tiles;  // pieces a group; across a workgroup; groups a workgroup or workgroups a group; tiles a row
    int chunk, chunks;                  // positions a workgroup, workgroups a sequence
};
struct SpanPlace {
    int b, chunk, part, first;  // first group
    int tx, ty, ly, local, k;   // this thread's group (of the workgroup's) and piece of it
    bool is;
};
__device__ __forceinline__ SpanPlace span_place(const Span& p, const NormIn& in, unsigned block) {
    SpanPlace m;
    const unsigned rest = block / p.tiles, tile = block - rest * p.tiles;
    m.b = rest / p.chunks;
    m.chunk = rest - m.b * p.chunks;
    m.part = p.parts > 1 ? tile % p.parts : 0;
    m.first = p.parts > 1 ? tile / p.parts : tile * p.groups;
    m.tx = threadIdx.x % p.lx;
    m.ty = threadIdx.x / p.lx;
    m.ly = 256 / p.lx;
    m.local = p.parts > 1 ? 0 : m.tx / p.ppg;
    m.k = p.parts > 1 ? m.part * p.lx + m.tx : m.tx - m.local * p.ppg;
    m.is = m.local < p.groups && m.first + m.local < in.G && m.k < p.ppg;
    return m;
}
// Values of a group's part at one position.
template <int W> __device__ __forceinline__ int part_width(const Span& p, int part, int C) {
    const int from = part * p.lx * W, to = from + p.lx * W;
    return p.parts == 1 ? C : (to < C ? to : C) - from;
}

// What has gone into lds[0 .. lx) is joined group by group: the first of a group's threads has it (threads of the first row of positions call with `mine`).
template <typename V, typename F> __device__ __forceinline__ void join_groups(V* lds, V& mine, const Span& p, const SpanPlace& my, F joined) {
    const int in_group = p.parts > 1 ? my.tx : my.k, size = p.parts > 1 ? p.lx : p.ppg;
    int k = 1;
    while (k < size) k *= 2;
    for (k /= 2; k >= 1; k /= 2) {
        __syncthreads();
        if (my.ty == 0 && my.local < p.groups && in_group < k && in_group + k < size) lds[my.tx] = mine = joined(mine, lds[my.tx + k]);
    }
}

// Joins the entries of the workgroup's groups, `threads` of them side by side: of(local group, entry) in ascending entries for each thread, then halves.  The results stand in
// lds[group * per], per threads a group.
template <typename V, typename Of, typename F> __device__ __forceinline__ int join_entries(V* lds, const Span& p, int first, int G, int64_t entries, const V& none, Of of, F joined) {
    int many = 1;
    while (many < p.groups) many *= 2;
    const int per = 256 / many, g = threadIdx.x / per, t = threadIdx.x - g * per;
    V v = none;
    if (g < p.groups && first + g < G)
        for (int64_t e = t; e < entries; e += per) v = joined(v, of(g, e));
    lds[threadIdx.x] = v;
    for (int k = per / 2; k >= 1; k /= 2) {
        __syncthreads();
        if (t < k) lds[threadIdx.x] = v = joined(v, lds[threadIdx.x + k]);
    }
    __syncthreads();
    return per;
}

// Moments of every group's part over a chunk: [B][G][chunks][parts][2] (mean, M; the count follows from the lengths).
constexpr int kBatch = 4;  // positions in flight
static_assert(kMaxPositions - 1 + kBatch * 256 < int64_t{1} << 31, "where a thread's next turn begins fits 32 bits");
template <typename T, int W>
__global__ __launch_bounds__(256) void moments_kernel(NormIn in, Span p, float* __restrict__ made) {
    __shared__ Moments lds[256];
    const SpanPlace my = span_place(p, in, blockIdx.x);
    const int len = length_at(in.lengths, my.b, in.N), begin = my.chunk * p.chunk, stop = len - begin < p.chunk ? len : begin + p.chunk;
    if (begin >= len) return;  // nobody looks at these
    const Place at = Place::of<W>(my.is ? (my.first + my.local) * p.ppg + my.k : 0, p.ppg, in.D / in.G);
    Moments m{0.0f, 0.0f, 0.0f};
    Part<T, W> v[kBatch];
    const auto fetch = [&](int l) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) v[u].load(line<T>(in.x, my.b, or_last(l, u * my.ly, stop)) + at.c, W);
    };
    int l = begin + my.ty;
    fetch(l);
    for (; l < stop; l += kBatch * my.ly) {
        float x[kBatch][W], s = 0.0f, q = 0.0f;
        int rows = 0;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            v[u].get(x[u]);
            rows += l + u * my.ly < stop;
        }
        fetch(l + kBatch * my.ly);
        if (rows == kBatch && at.skip == 0) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
#pragma unroll
                for (int j = 0; j < W; ++j) s += x[u][j];
            const float mean = s * (1.0f / (kBatch * W));
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
#pragma unroll
                for (int j = 0; j < W; ++j) q = fmaf(x[u][j] - mean, x[u][j] - mean, q);
            m = join(m, {kBatch * W, mean, q});
        } else {
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
#pragma unroll
                for (int j = 0; j < W; ++j) s += u < rows && j >= at.skip ? x[u][j] : 0.0f;
            const float n = static_cast<float>(rows * (W - at.skip)), mean = s / n;
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
#pragma unroll
                for (int j = 0; j < W; ++j) q = u < rows && j >= at.skip ? fmaf(x[u][j] - mean, x[u][j] - mean, q) : q;
            m = join(m, {n, mean, q});
        }
    }
    if (!my.is) m = {0.0f, 0.0f, 0.0f};
    lds[threadIdx.x] = m;
    for (int k = 128; k >= p.lx; k /= 2) {  // lx is a power of two
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < k) lds[threadIdx.x] = m = join(m, lds[threadIdx.x + k]);
    }
    join_groups(lds, m, p, my, join);
    if (my.ty == 0 && my.is && (p.parts > 1 ? my.tx : my.k) == 0) {
        float* to = made + (((static_cast<int64_t>(my.b) * in.G + my.first + my.local) * p.chunks + my.chunk) * p.parts + my.part) * 2;
        to[0] = m.mean;
        to[1] = m.m2;
    }
}

// (mean, rstd) of this thread's group: given, or joined from the moments.  keep: written there.
template <int W> __device__ __forceinline__ void span_stats(const NormIn& in, const Span& p, const SpanPlace& my, int len, const float* given, const float* made, float* keep,
                                                            Moments* lds, float& mean, float& rstd) {
    mean = rstd = 0.0f;
    if (given) {
        if (my.is) {
            mean = given[(static_cast<int64_t>(my.b) * in.G + my.first + my.local) * 2];
            rstd = given[(static_cast<int64_t>(my.b) * in.G + my.first + my.local) * 2 + 1];
        }
        return;
    }
    const int chunks = len > 0 ? (len - 1) / p.chunk + 1 : 0, C = in.D / in.G;
    const int per = join_entries(lds, p, my.first, in.G, static_cast<int64_t>(chunks) * p.parts, Moments{0.0f, 0.0f, 0.0f}, [&](int g, int64_t e) {
        const int k = static_cast<int>(e / p.parts), part = static_cast<int>(e - static_cast<int64_t>(k) * p.parts);
        const int rows = len - k * p.chunk < p.chunk ? len - k * p.chunk : p.chunk;
        const float* from = made + ((static_cast<int64_t>(my.b) * in.G + my.first + g) * p.chunks * p.parts + e) * 2;
        return Moments{static_cast<float>(rows) * part_width<W>(p, part, C), from[0], from[1]};
    }, join);
    if (my.is) {
        const Moments m = lds[my.local * per];
        mean = m.mean;
        rstd = len > 0 ? __builtin_amdgcn_rsqf(m.m2 / m.n + in.eps) : 0.0f;
        if (keep && my.chunk == 0 && my.ty == 0 && my.k == 0) {
            keep[(static_cast<int64_t>(my.b) * in.G + my.first + my.local) * 2] = mean;
            keep[(static_cast<int64_t>(my.b) * in.G + my.first + my.local) * 2 + 1] = rstd;
        }
    }
}

// Sums over parts of dweight and dbias, [parts][2][D]: workgroups of 16 channels of one of the two, HIGH threads a channel.
template <int HIGH> __device__ __forceinline__ void channel_sums(const float* partial, int64_t parts, int D, int64_t block, float* dweight, float* dbias, float* lds) {
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4, k = block & 1;
    const int64_t ch = (block >> 1) * 16 + x;
    float* to = k ? dbias : dweight;
    float s = 0.0f;
    if (to && ch < D)
#pragma unroll 4
        for (int64_t q = y; q < parts; q += HIGH) s += partial[(q * 2 + k) * D + ch];
    lds[threadIdx.x] = s;
    for (int h = HIGH / 2; h >= 1; h /= 2) {
        __syncthreads();
        if (y < h) lds[threadIdx.x] = s = s + lds[threadIdx.x + 16 * h];
    }
    if (y == 0 && to && ch < D) to[ch] = s;
}
__global__ __launch_bounds__(1024) void channel_sums_kernel(const float* __restrict__ partial, int64_t parts, int D, float* __restrict__ dweight, float* __restrict__ dbias) {
    __shared__ float lds[1024];
    channel_sums<64>(partial, parts, D, blockIdx.x, dweight, dbias, lds);
}
int64_t channel_blocks(int D) { return 2 * static_cast<int64_t>((D - 1) / 16 + 1); }

struct Sum2 { float a, b; };
__device__ __forceinline__ Sum2 add(const Sum2& x, const Sum2& y) { return {x.a + y.a, x.b + y.b}; }

struct ApplyRun {
    const float *given, *made;  // statistics, or the moments they come from
    float* stats;               // forwards: to be kept, or null
    const float* sums;          // GRAD: [B][G][chunks][parts][2]
    const float* partial;       // GRAD: [B * chunks][2][D], summed by the first `extra` workgroups
    int64_t extra;
    float *dweight, *dbias;
    bool stream;
};
template <typename T, int W, bool GRAD>
__global__ __launch_bounds__(256) void apply_kernel(NormIn in, AnyRows dout, Span p, ApplyRun r, T* __restrict__ out) {
    __shared__ Moments lds[256];
    if (GRAD && blockIdx.x < r.extra) {
        channel_sums<16>(r.partial, static_cast<int64_t>(in.B) * p.chunks, in.D, blockIdx.x, r.dweight, r.dbias, reinterpret_cast<float*>(lds));
        return;
    }
    const SpanPlace my = span_place(p, in, blockIdx.x - static_cast<unsigned>(GRAD ? r.extra : 0));
    const int len = length_at(in.lengths, my.b, in.N), begin = my.chunk * p.chunk, stop = in.N - begin < p.chunk ? in.N : begin + p.chunk;
    const int end = len < begin ? begin : len < stop ? len : stop;
    const Place at = Place::of<W>(my.is ? (my.first + my.local) * p.ppg + my.k : 0, p.ppg, in.D / in.G);
    Part<T, W> v[kBatch], d[GRAD ? kBatch : 1];
    const auto fetch = [&](int l) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int at_l = or_last(l, u * my.ly, end);
            v[u].load(line<T>(in.x, my.b, at_l) + at.c, W);
            if (GRAD) d[u].load(line<T>(dout, my.b, at_l) + at.c, W);
        }
    };
    int l = begin + my.ty;
    if (end > begin) fetch(l);  // on their way while the sums are joined
    float w[W], bias[W];
    weights_of<W>(in, at.c, w, bias);
    float mean, rstd, s1 = 0.0f, s2 = 0.0f;
    span_stats<W>(in, p, my, len, r.given, r.made, GRAD ? nullptr : r.stats, lds, mean, rstd);
    if (GRAD) {
        __syncthreads();
        Sum2* two = reinterpret_cast<Sum2*>(lds);
        const int chunks = len > 0 ? (len - 1) / p.chunk + 1 : 0;
        const int per = join_entries(two, p, my.first, in.G, static_cast<int64_t>(chunks) * p.parts, Sum2{0.0f, 0.0f}, [&](int g, int64_t e) {
            const float* from = r.sums + ((static_cast<int64_t>(my.b) * in.G + my.first + g) * p.chunks * p.parts + e) * 2;
            return Sum2{from[0], from[1]};
        }, add);
        if (my.is && len > 0) {
            const float n = static_cast<float>(len) * (in.D / in.G);
            s1 = two[my.local * per].a / n;
            s2 = two[my.local * per].b / n;
        }
    }
    if (!my.is) return;
    T* o = out + static_cast<int64_t>(my.b) * in.N * in.D + at.c;
    float scale[W];
#pragma unroll
    for (int j = 0; j < W; ++j) scale[j] = rstd * w[j];
    for (; l < end; l += kBatch * my.ly) {
        float x[kBatch][W], dy[GRAD ? kBatch : 1][W];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            v[u].get(x[u]);
            if (GRAD) d[u].get(dy[u]);
        }
        fetch(l + kBatch * my.ly);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const float away = x[u][j] - mean;
                if (GRAD) {
                    const float hat = away * rstd;
                    x[u][j] = fmaf(in.silu ? dy[u][j] * dsilu(fmaf(hat, w[j], bias[j])) : dy[u][j], scale[j], -rstd * fmaf(hat, s2, s1));
                } else {
                    const float y = fmaf(away, scale[j], bias[j]);
                    x[u][j] = in.silu ? silu(y) : y;
                }
            }
            if (l + u * my.ly < end) {
                T* to = o + static_cast<int64_t>(l + u * my.ly) * in.D;
                if (r.stream) Part<T, W>::template put<true>(to, W, x[u]);
                else Part<T, W>::put(to, W, x[u]);
            }
        }
    }
    const float zero[W] = {};
    for (l = end + my.ty; l < stop; l += my.ly) Part<T, W>::put(o + static_cast<int64_t>(l) * in.D, W, zero);
}

// Sums of dy hat and dy over a chunk's positions, channel by channel, [B * chunks][2][D] (partial may be null), and weighed, of a group's part: [B][G][chunks][parts][2].
// ALONE: every position has its own statistics, B is 1 and N all positions, and there are no groups' sums.
template <typename T, int W, bool ALONE>
__global__ __launch_bounds__(256) void columns_kernel(NormIn in, AnyRows dout, Span p, const float* __restrict__ given, const float* __restrict__ made,
                                                      float* __restrict__ partial, float* __restrict__ sums) {
    __shared__ union { Moments m[256]; float f[256 * 2 * W]; Sum2 s[256]; } lds;
    const SpanPlace my = span_place(p, in, blockIdx.x);
    const int len = ALONE ? in.B * in.N : length_at(in.lengths, my.b, in.N), begin = my.chunk * p.chunk;
    const int stop = len - begin < p.chunk ? len : begin + p.chunk;
    const Place at = Place::of<W>(my.is ? (my.first + my.local) * p.ppg + my.k : 0, p.ppg, in.D / in.G);
    float w[W], bias[W], dw[W] = {}, db[W] = {}, mean = 0.0f, rstd = 0.0f;
    weights_of<W>(in, at.c, w, bias);
    Part<T, W> v[kBatch], d[kBatch];
    float means[ALONE ? kBatch : 1], rstds[ALONE ? kBatch : 1];
    bool on[kBatch];
    const auto fetch = [&](int l) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            on[u] = my.is && before(l, u * my.ly, stop);
            const int pos = or_last(l, u * my.ly, stop), b = ALONE ? pos / in.N : my.b, row = ALONE ? pos - b * in.N : pos;
            if (ALONE) {
                on[u] = on[u] && row < length_at(in.lengths, b, in.N);
                means[u] = given[(static_cast<int64_t>(pos) * in.G + at.group) * 2];
                rstds[u] = given[(static_cast<int64_t>(pos) * in.G + at.group) * 2 + 1];
            }
            if (!ALONE || on[u]) {
                v[u].load(line<T>(in.x, b, row) + at.c, W);
                d[u].load(line<T>(dout, b, row) + at.c, W);
            }
        }
    };
    int l = begin + my.ty;
    if (begin < stop) fetch(l);  // on their way while the statistics are joined
    if (!ALONE) span_stats<W>(in, p, my, len, given, made, nullptr, lds.m, mean, rstd);
    for (; l < stop; l += kBatch * my.ly) {
        float x[kBatch][W], dy[kBatch][W], hats[ALONE ? kBatch : 1][2];
        bool is[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            v[u].get(x[u]);
            d[u].get(dy[u]);
            is[u] = on[u];
            if (ALONE) {
                hats[u][0] = means[u];
                hats[u][1] = rstds[u];
            }
        }
        fetch(l + kBatch * my.ly);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const float hat = (x[u][j] - (ALONE ? hats[u][0] : mean)) * (ALONE ? hats[u][1] : rstd);
                const float g = in.silu ? dy[u][j] * dsilu(fmaf(hat, w[j], bias[j])) : dy[u][j];
                dw[j] = is[u] ? fmaf(g, hat, dw[j]) : dw[j];
                db[j] = is[u] ? db[j] + g : db[j];
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < W; ++j) {
        lds.f[(2 * j) * 256 + threadIdx.x] = dw[j];
        lds.f[(2 * j + 1) * 256 + threadIdx.x] = db[j];
    }
    for (int h = my.ly / 2; h >= 1; h /= 2) {
        __syncthreads();
        if (my.ty < h) {
#pragma unroll
            for (int j = 0; j < 2 * W; ++j) lds.f[j * 256 + threadIdx.x] += lds.f[j * 256 + threadIdx.x + h * p.lx];
        }
    }
    Sum2 mine{0.0f, 0.0f};
    if (my.ty == 0 && my.is) {
        float* to = partial ? partial + (static_cast<int64_t>(my.b) * p.chunks + my.chunk) * 2 * in.D + at.c : nullptr;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            if (j < at.skip) continue;
            const float s_hat = lds.f[(2 * j) * 256 + threadIdx.x], s = lds.f[(2 * j + 1) * 256 + threadIdx.x];
            if (to) {
                to[j] = s_hat;
                to[in.D + j] = s;
            }
            mine.a = fmaf(w[j], s, mine.a);
            mine.b = fmaf(w[j], s_hat, mine.b);
        }
    }
    if (ALONE) return;
    __syncthreads();
    if (my.ty == 0) lds.s[my.tx] = mine;
    join_groups(lds.s, mine, p, my, add);
    if (my.ty == 0 && my.is && (p.parts > 1 ? my.tx : my.k) == 0) {
        float* to = sums + (((static_cast<int64_t>(my.b) * in.G + my.first + my.local) * p.chunks + my.chunk) * p.parts + my.part) * 2;
        to[0] = mine.a;
        to[1] = mine.b;
    }
}

// ---- launches -------------------------------------------------------------------------------------------------

int piece_width(int dtype, int C) {
    int w = dtype ? 8 : 4;
    while (w > C) w /= 2;
    return w;
}

constexpr int kMostPieces = 4;  // a lane's, in registers

bool alone_fits(int ppg) { return ppg <= 256 * kMostPieces; }
// Lanes a team and pieces a lane: one each as long as a wave has the lanes; 3 pieces where that leaves fewer of them without one; a workgroup a team where a
// wave's lanes would take more than 16 channels each.
void team_of(int ppg, int W, int& team, int& pieces) {
    team = 1;
    while (team < 64 && team < ppg) team *= 2;
    if (ppg > 64 * 16 / W) team = 256;
    pieces = (ppg - 1) / team + 1;
    if (pieces == 1 && team >= 4 && team <= 64 && 3 * (team / 4) >= ppg) {
        team /= 4;
        pieces = 3;
    }
}

// Workgroups: as many as the chip holds at once by the registers that they take, then they take their positions in turn (a second round for a few of them costs as
// much as the first; B=128 N=128 D=1001 in seven groups, float, ragged, gradient in 768 workgroups of three waves a SIMD 90 us for the whole training step,
// in 1024 103).
Alone alone_plan(int dtype, int B, int N, int D, int G, bool grad, int& pieces) {
    Alone p;
    const int C = D / G, W = piece_width(dtype, C);
    p.ppg = (C - 1) / W + 1;
    team_of(p.ppg, W, p.team, pieces);
    p.groups = 1;
    while (p.team < 64 && p.groups < 64 / p.team && p.groups < G) p.groups *= 2;
    p.tiles = (G - 1) / p.groups + 1;
    const int64_t rows = p.team > 64 ? 1 : 4 * (64 / p.team / p.groups), all = (static_cast<int64_t>(B) * N + rows - 1) / rows;
    // Waves a SIMD of the gradient: 4 up to two pieces of 4 channels (or one of 8), 3 of three pieces of 4 and of two of 8, 2, 1.  (Of two pieces of 8 only where every lane has
    // its own: others take 172 registers and run two waves a SIMD, and 768 workgroups are half as many again as the chip holds: 64 x 512 x 1000 in one group, bfloat16,
    // 77 us, in 512 workgroups 63; 1024 channels 58.)
    const int registers = pieces * (W == 8 ? 2 : 1);
    int64_t most = (!grad || registers <= 2 ? 1024 : registers == 3 || (registers == 4 && W == 8) ? 768 : registers <= 6 ? 512 : 256) / p.tiles;
    if (most < 1) most = 1;
    p.blocks = all < most ? all : most;
    return p;
}

Span span_plan(int dtype, int B, int N, int D, int G) {
    Span p;
    const int C = D / G, W = piece_width(dtype, C);
    p.ppg = (C - 1) / W + 1;
    const int64_t pieces = static_cast<int64_t>(p.ppg) * G;
    p.parts = (p.ppg - 1) / 256 + 1;
    p.lx = 1;
    while (p.lx < 64 && p.lx < pieces) p.lx *= 2;
    while (p.lx < 256 && p.lx < p.ppg) p.lx *= 2;
    // wider where groups leave fewer threads without a piece
    for (int lx = 2 * p.lx; p.parts == 1 && lx <= 256 && lx / 2 < pieces; lx *= 2)
        if (lx / p.ppg * p.ppg * p.lx * 8 > p.lx / p.ppg * p.ppg * lx * 9) p.lx = lx;
    p.groups = p.parts > 1 ? 1 : p.lx / p.ppg;
    p.tiles = p.parts > 1 ? G * p.parts : (G - 1) / p.groups + 1;
    const int least = kBatch * (256 / p.lx);  // a chunk's positions: as many as keep 512 workgroups, at most 16 batches of a thread
    p.chunk = 16 * least;
    while (p.chunk > least && static_cast<int64_t>(B) * p.tiles * ((N - 1) / p.chunk + 1) < 512) p.chunk /= 2;
    p.chunks = (N - 1) / p.chunk + 1;
    return p;
}

// Whether a sequence's groups fit registers.  At least 64 bytes of a row a workgroup, more where groups leave fewer lanes without a piece; as many threads as hold
// the positions in R pieces.  Runs of sixteen tiles, of two where that would leave XCDs without one.  Measured, us, bfloat16, runs of 1 / 2 / 16 tiles of 64 bytes, of 16 of
// 128: 64 x 512 x 1024 in 32 groups 133 / 28 / 29 / 31 (4.7 TB/s; two passes 40), with its gradient - / 116 / 109 / 112 (two passes 117), 256 x 512 x 1024 - / 149 / 123 / 117,
// gradient of 20 x 500 x 2048 in 64 groups - / 72 / 73 / 79.  Over kHeldBytes threads hold eight pieces in one go: fewer and larger workgroups.
constexpr int64_t kHeldBytes = int64_t{16} << 20;
bool held_plan(int dtype, int B, int N, int D, int G, Held& p) {
    const bool large = static_cast<int64_t>(B) * N * D * (dtype ? 2 : 4) > kHeldBytes;
    const int C = D / G, W = piece_width(dtype, C), line = 64 / (W * (dtype ? 2 : 4));
    p.ppg = (C - 1) / W + 1;
    if (p.ppg > 512) return false;
    const int64_t pieces = static_cast<int64_t>(p.ppg) * G;
    int least = 1;
    while (least < p.ppg || (least < line && least < pieces)) least *= 2;
    p.lx = least;
    for (int lx = 2 * least; lx <= 4 * least && lx <= 256; lx *= 2)  // (never across more than a row has)
        if (lx / 2 < pieces && lx / p.ppg * p.ppg * p.lx > p.lx / p.ppg * p.ppg * lx * 9 / 8) p.lx = lx;
    p.groups = p.lx / p.ppg;
    p.tiles = (G - 1) / p.groups + 1;
    p.run = static_cast<int64_t>(B) * p.tiles >= 256 ? 16 : 2;
    for (const int most : {2, 4, 8})
        for (p.threads = 256; p.threads <= (most > 4 ? 512 : 1024); p.threads *= 2) {
            if (p.threads < p.lx || (N - 1) / (p.threads / p.lx) + 1 > most) continue;
            if (large && most < 8) continue;
            p.pieces = most;
            return true;
        }
    return false;
}

// two floats a group's part and chunk
size_t entries_bytes(const Span& p, int B, int G) { return up256(static_cast<size_t>(B) * G * p.chunks * p.parts * 8); }
size_t stats_bytes(int64_t units) { return up256(static_cast<size_t>(units) * 8); }
size_t partial_bytes(int64_t parts, int D) { return up256(static_cast<size_t>(parts) * 2 * D * 4); }

template <typename T, int W, bool GRAD>
hipError_t alone_of(const NormIn& in, AnyRows dout, const Alone& p, int pieces, const float* given, void* out, float* stats, float* partial, hipStream_t st) {
    if (!fits(p.blocks * p.tiles, 256)) return hipErrorInvalidValue;
    const bool exact = in.D / in.G == p.team * pieces * W;
    auto kernel = exact ? alone_kernel<T, W, 1, GRAD, true, false> : alone_kernel<T, W, 1, GRAD, false, false>;
    if constexpr (W == Wide<T>::V) {  // narrower pieces are at most two a group
        if (p.team > 64) {
            kernel = pieces == 1 ? alone_kernel<T, W, 1, GRAD, false, true> : pieces == 2 ? alone_kernel<T, W, 2, GRAD, false, true>
                     : pieces == 3 ? alone_kernel<T, W, 3, GRAD, false, true> : alone_kernel<T, W, 4, GRAD, false, true>;
        } else {
            if (pieces == 2) kernel = exact ? alone_kernel<T, W, 2, GRAD, true, false> : alone_kernel<T, W, 2, GRAD, false, false>;
            if (pieces == 3) kernel = alone_kernel<T, W, 3, GRAD, false, false>;
            if constexpr (W == 4)
                if (pieces == 4) kernel = exact ? alone_kernel<T, W, 4, GRAD, true, false> : alone_kernel<T, W, 4, GRAD, false, false>;
        }
    }
    kernel<<<static_cast<unsigned>(p.blocks * p.tiles), 256, 0, st>>>(in, dout, p, given, static_cast<T*>(out), stats, partial);
    return hipGetLastError();
}

template <typename T, int W, bool GRAD>
hipError_t held_of(const NormIn& in, AnyRows dout, const Held& p, const float* given, void* out, float* stats, float* partial, hipStream_t st) {
    const int64_t round = 8 * p.run, blocks = (static_cast<int64_t>(in.B) * p.tiles + round - 1) / round * round;
    if (!fits(blocks, p.threads)) return hipErrorInvalidValue;
    const auto kernel = p.pieces == 2 ? held_kernel<T, W, 2, GRAD> : p.pieces == 4 ? held_kernel<T, W, 4, GRAD> : held_kernel<T, W, 8, GRAD>;
    const int entries = p.threads / 64 * (p.lx < 64 ? p.lx : 64);
    int floats = p.threads + p.lx;
    if (GRAD && floats < W * entries) floats = W * entries;
    if (floats < 2 * p.lx) floats = 2 * p.lx;
    kernel<<<static_cast<unsigned>(blocks), p.threads, sizeof(float) * floats, st>>>(in, dout, p, given, static_cast<T*>(out), stats, partial);
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
        const Alone p = alone_plan(dtype, in.B, in.N, in.D, in.G, false, pieces);
        if (alone_fits(p.ppg)) return alone_of<T, W, false>(in, {}, p, pieces, nullptr, o.out, o.stats, nullptr, st);
        if constexpr (W == Wide<T>::V) {
            const int64_t units = static_cast<int64_t>(in.B) * in.N * in.G;
            wide_kernel<T, W, false><<<static_cast<unsigned>(units < kWideBlocks ? units : kWideBlocks), 256, 0, st>>>(in, {}, p.ppg, nullptr, static_cast<T*>(o.out), o.stats);
        }
        return hipGetLastError();
    }
    Held h;
    if (held_plan(dtype, in.B, in.N, in.D, in.G, h)) return held_of<T, W, false>(in, {}, h, nullptr, o.out, o.stats, nullptr, st);
    const Span p = span_plan(dtype, in.B, in.N, in.D, in.G);
    const int64_t blocks = static_cast<int64_t>(in.B) * p.chunks * p.tiles;
    if (!fits(blocks, 256)) return hipErrorInvalidValue;
    float* made = static_cast<float*>(ws);
    moments_kernel<T, W><<<static_cast<unsigned>(blocks), 256, 0, st>>>(in, p, made);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const ApplyRun r{nullptr, made, o.stats, nullptr, nullptr, 0, nullptr, nullptr, past_caches(static_cast<int64_t>(in.B) * in.N * in.D * static_cast<int64_t>(sizeof(T)))};
    apply_kernel<T, W, false><<<static_cast<unsigned>(blocks), 256, 0, st>>>(in, {}, p, r, static_cast<T*>(o.out));
    return hipGetLastError();
}

hipError_t launch_channel_sums(const float* partial, int64_t parts, const NormIn& in, const Outs& o, hipStream_t st) {
    channel_sums_kernel<<<static_cast<unsigned>(channel_blocks(in.D)), 1024, 0, st>>>(partial, parts, in.D, o.dweight, o.dbias);
    return hipGetLastError();
}

template <typename T, int W>
hipError_t norm_grad_of(int dtype, AnyRows dout, const NormIn& in, const float* stats, const Outs& o, void* ws, hipStream_t st) {
    char* room = static_cast<char*>(ws);
    const bool sums = o.dweight || o.dbias;
    if (in.alone) {
        int pieces;
        const Alone p = alone_plan(dtype, in.B, in.N, in.D, in.G, true, pieces);
        float* partial = reinterpret_cast<float*>(room);
        if (alone_fits(p.ppg)) {
            if (const hipError_t e = alone_of<T, W, true>(in, dout, p, pieces, stats, o.out, nullptr, sums ? partial : nullptr, st); e != hipSuccess || !sums) return e;
            return launch_channel_sums(partial, p.blocks, in, o, st);
        }
        if constexpr (W == Wide<T>::V) {
            const int64_t units = static_cast<int64_t>(in.B) * in.N * in.G;
            const Span q = span_plan(dtype, 1, in.B * in.N, in.D, in.G);
            if (!fits(static_cast<int64_t>(q.chunks) * q.tiles, 256)) return hipErrorInvalidValue;
            float* made = reinterpret_cast<float*>(room + partial_bytes(q.chunks, in.D));
            wide_kernel<T, W, true><<<static_cast<unsigned>(units < kWideBlocks ? units : kWideBlocks), 256, 0, st>>>(in, dout, p.ppg, stats, static_cast<T*>(o.out), stats ? nullptr : made);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess || !sums) return e;
            columns_kernel<T, W, true><<<static_cast<unsigned>(q.chunks * q.tiles), 256, 0, st>>>(in, dout, q, stats ? stats : made, nullptr, partial, nullptr);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
            return launch_channel_sums(partial, q.chunks, in, o, st);
        }
        return hipErrorInvalidValue;
    }
    Held h;
    if (held_plan(dtype, in.B, in.N, in.D, in.G, h)) {
        float* partial = reinterpret_cast<float*>(room);
        if (const hipError_t e = held_of<T, W, true>(in, dout, h, stats, o.out, nullptr, sums ? partial : nullptr, st); e != hipSuccess || !sums) return e;
        return launch_channel_sums(partial, in.B, in, o, st);
    }
    const Span p = span_plan(dtype, in.B, in.N, in.D, in.G);
    const int64_t blocks = static_cast<int64_t>(in.B) * p.chunks * p.tiles, extra = sums ? channel_blocks(in.D) : 0;
    if (!fits(blocks + extra, 256)) return hipErrorInvalidValue;
    float* partial = reinterpret_cast<float*>(room);
    room += partial_bytes(static_cast<int64_t>(in.B) * p.chunks, in.D);
    float* of_groups = reinterpret_cast<float*>(room);
    room += entries_bytes(p, in.B, in.G);
    float* made = reinterpret_cast<float*>(room);
    if (!stats) {
        moments_kernel<T, W><<<static_cast<unsigned>(blocks), 256, 0, st>>>(in, p, made);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    columns_kernel<T, W, false><<<static_cast<unsigned>(blocks), 256, 0, st>>>(in, dout, p, stats, made, sums ? partial : nullptr, of_groups);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const ApplyRun r{stats, made, nullptr, of_groups, partial, extra, o.dweight, o.dbias, past_caches(static_cast<int64_t>(in.B) * in.N * in.D * static_cast<int64_t>(sizeof(T)))};
    apply_kernel<T, W, true><<<static_cast<unsigned>(blocks + extra), 256, 0, st>>>(in, dout, p, r, static_cast<T*>(o.out));
    return hipGetLastError();
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
    Held h;
    if (alone || held_plan(dtype, B, N, D, G, h)) return 0;
    return entries_bytes(span_plan(dtype, B, N, D, G), B, G);
}

size_t norm_grad_workspace(int dtype, int B, int N, int D, int G, bool alone) {
    if (alone) {
        int pieces;
        const Alone p = alone_plan(dtype, B, N, D, G, true, pieces);
        if (alone_fits(p.ppg)) return partial_bytes(p.blocks, D);
        return partial_bytes(span_plan(dtype, 1, B * N, D, G).chunks, D) + stats_bytes(static_cast<int64_t>(B) * N * G);
    }
    Held h;
    if (held_plan(dtype, B, N, D, G, h)) return partial_bytes(B, D);
    const Span p = span_plan(dtype, B, N, D, G);
    return partial_bytes(static_cast<int64_t>(B) * p.chunks, D) + 2 * entries_bytes(p, B, G);
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
