// Group norm with an activation, channels last, forward and backward: the kernels and their launches for one element type (group_norm_f32.hip,
// group_norm_bf16.hip, group_norm_f16.hip).
//
// The work is cut into tiles of whole groups, a 128-byte line wide or a little more (a part of a line in one launch), and a tile's pixels into chunks, one to a workgroup.  A
// thread keeps one piece of V channels (up to 16 bytes) and walks down the chunk's pixels, so that scale, bias and statistics of its channels stay in
// registers.  Statistics need all of a group before the first output: a map whose tiles fit the registers of a workgroup each takes one launch and is read once;
// all others take two, of which one leaves each chunk's part and the other joins the parts of its groups in a fixed order and reads the map again.
//
// Bound by memory where the map is large: 4 images of 256 x 256 pixels and 128 channels in bf16 take 37.6 us (15.6 + 22.5, 201 MB read and written at 5.4 TB/s; read
// once, at the rate of a large copy, 26.2), their backward pass 60.2 us (30.3 + 32.3, 335 MB at 5.6 TB/s; 39.2).  The second reading comes from the memory-side cache in part.  Vector
// instructions (silu: 20 slots an element forward, 43 backward, an exponential and an inverse four each) are 17 and 36 us of that and run beside the memory.  Bound
// by latency where it is small: 4 images of 32 x 32 and 512 channels 7.9 us.
//
// Tried and not kept: one launch for large maps, whose chunks stay in registers while the workgroups of a tile send each other their parts through memory.  The map
// is read once, but loading, arithmetic, exchange (3 .. 15 us: chunks^2 reads of few lines) and storing follow each other in lockstep: 52.6 us for the first map above, 98.6
// backward.
#pragma once

#include "qrm_train.h"

#include <algorithm>
#include <type_traits>

namespace qrm {
namespace {

constexpr int kThreads = kNormThreads, kMaxThreads = kNormMaxThreads;
constexpr uint32_t kDies = 8; // workgroups go to the dies in turn, each with an L2 of its own

struct NormArgs {
    const void *x, *dy;
    void *y, *dx;
    const float *gamma, *beta;
    float *mean, *rstd, *dgamma, *dbeta;
    float2 *part;          // two launches: [N][G][parts]: (mean, sum of squares about it); backward (sum gamma dz, sum gamma dz h)
    float2 *chan;          // backward: [N * parts][C]: (sum dz, sum dz h); null: not wanted, or written at once
    int64_t N, P;
    int64_t xp, xn, yp, yn;
    int C, G, D;
    int ct, tiles, chunks, rpar; // this launch's cut; rpar: pixels side by side
    int side;                    // neighbouring tiles that lie in the same lines
    uint32_t turned;             // .. and the workgroups that are numbered for it
    int parts, parts_rpar;       // the first launch's chunks and pixels side by side
    int act;
    float eps;
};

// What a workgroup is about: its image, channels and pixels, and its threads' places in them.
struct Tile {
    int64_t n, step;       // image, distance of a thread's pixels
    int base, extra;       // pixels at a place side by side: `base`, one more at the first `extra` places
    int t, s;              // tile, chunk
    int c0, g0, groups;    // first channel and group, number of groups
    int cols, rpar;        // pieces across, pixels side by side (as many in the last, narrower tile)
    int r, col;            // this thread's; r >= rpar: none
};

// Pixels of a chunk that the threads at `r` of those side by side take: the chunks take turns, so that all workgroups move down the map together.
__device__ __forceinline__ int pixels_at(const Tile &t, int r) { return t.base + (r < t.extra); }

// The tiles of the same pixels lie side by side in the grid; those that share lines are numbered kDies apart, so that one die's cache serves them: 4 images of 1024
// pixels and 512 channels, tiles of a quarter line, 7.9 us against 8.6, of 2048 pixels 11.1 against 15.0.
template <int V> __device__ __forceinline__ Tile find_tile(const NormArgs &a)
{
    Tile t;
    uint32_t b = blockIdx.x;
    if (b < a.turned) {
        const uint32_t k = b / kDies, set = kDies * a.side;
        b = b / set * set + b % kDies * a.side + k % a.side;
    }
    t.t = b % a.tiles;
    b /= a.tiles;
    t.s = b % a.chunks;
    t.n = b / a.chunks;
    t.c0 = t.t * a.ct;
    const int cw = min(a.ct, a.C - t.c0);
    t.g0 = t.c0 / a.D;
    t.groups = cw / a.D;
    t.cols = cw / V;
    t.rpar = a.rpar;
    t.r = threadIdx.x / t.cols;
    t.col = threadIdx.x % t.cols;
    const int64_t round = (int64_t)a.chunks * t.rpar, rest = a.P % round;
    t.base = (int)(a.P / round);
    t.extra = (int)max((int64_t)0, min((int64_t)t.rpar, rest - (int64_t)t.s * t.rpar));
    t.step = round;
    return t;
}

template <typename T, int V> __device__ __forceinline__ const T *x_at(const NormArgs &a, const Tile &t, int r)
{
    return (const T *)a.x + t.n * a.xn + ((int64_t)t.s * t.rpar + r) * a.xp + t.c0 + t.col * V;
}
template <int V> __device__ __forceinline__ int64_t y_offset(const NormArgs &a, const Tile &t, int r)
{
    return t.n * a.yn + ((int64_t)t.s * t.rpar + r) * a.yp + t.c0 + t.col * V;
}

// The thread's pieces of a chunk of up to R pixels side by side each; those that are not there are the chunk's first pixel.
template <typename T, int V, int R> __device__ __forceinline__ void read_chunk(const T *first, int64_t step, int r, int pixels, int64_t pitch, Words<T, V> (&x)[R])
{
    const T *p = first + r * pitch;
#pragma unroll
    for (int i = 0; i < R; ++i) x[i] = load_words<T, V>(i < pixels ? p + i * step : first);
}

// R pixels of a thread, `step` apart: the `top`-th from the first one on downwards (DOWN) or from the `top`-th on upwards; those outside 0 .. pixels-1 are the nearest
// inside.  p: the thread's first pixel, or any pixel of the chunk where it has none (pixels = 0).
template <typename T, int V, int R, bool DOWN> __device__ __forceinline__ void fetch(const T *p, int64_t step, int top, int pixels, Words<T, V> (&x)[R])
{
#pragma unroll
    for (int i = 0; i < R; ++i) x[i] = load_words<T, V>(p + max(0, DOWN ? top - 1 - i : min(top + i, pixels - 1)) * step);
}

constexpr int kLanes = 16; // lanes that join a group's columns

__device__ __forceinline__ float2 *part_at(const NormArgs &a, const Tile &t, int g, int s)
{
    return a.part + ((size_t)t.n * a.G + t.g0 + g) * a.parts + s;
}
// A lane's share of a group's parts (every `lanes`-th from `lane` on), several on their way at a time.  The first are asked for before the pixels are:
// what is waited for first has to be asked for first.
struct Parts {
    static constexpr int K = 4;
    const float2 *part;
    int parts, lane, lanes;
    float2 v[K];
    __device__ __forceinline__ void ask(int s)
    {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = part[min(s + k * lanes, parts - 1)];
    }
    __device__ __forceinline__ Parts(const float2 *p, int count, int l, int n) : part(p), parts(count), lane(l), lanes(n) { ask(l); }
    template <typename F> __device__ __forceinline__ void each(F use) // use(part, its index), in order
    {
        for (int s = lane; s < parts;) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (s + k * lanes < parts) use(v[k], s + k * lanes);
            s += K * lanes;
            if (s < parts) ask(s);
        }
    }
};
// How many lanes join a group of the tile: all threads have a part in it where they can.
__device__ __forceinline__ int lanes_for(int groups)
{
    int lanes = 64;
    while (lanes > 1 && groups * lanes > (int)blockDim.x) lanes /= 2;
    return lanes;
}

// ---------------------------------------------------------------- forward

// float2s of shared memory for W sums a thread and, where several pixels lie side by side, those over them: up to one a thread or one a column.
__host__ __device__ constexpr int sum_floats2(int threads, int W, int rpar) { return threads * W + (rpar == 1 ? 0 : W > 2 ? threads * W / 2 : threads); }

// Mean of `count` values and their squares about it; sets are joined by Chan's formula, so nothing cancels however far the mean
// lies from zero.
__device__ __forceinline__ void join_spread(float &mean, float &m2, float &count, float mean_b, float m2_b, float count_b)
{
    if (count_b > 0.f) {
        const float total = count + count_b, share = count_b * __builtin_amdgcn_rcpf(total), delta = mean_b - mean;
        mean = count > 0.f ? mean + delta * share : mean_b;
        m2 += m2_b + (count > 0.f ? delta * delta * (count * share) : 0.f);
        count = total;
    }
}

template <int W> struct Spread {
    float mean[W], m2[W], count;
};

// Joins up to R pixels' values: their own mean and squares first, exact to rounding.
template <typename T, int V, int W, int R> __device__ __forceinline__ void spread_batch(Spread<W> &s, Words<T, V> (&x)[R], int pixels)
{
    if (pixels <= 0) return;
    const float k = (float)(min(pixels, R) * (V / W)), inv = 1.f / k;
    float mean[W], m2[W];
#pragma unroll
    for (int w = 0; w < W; ++w) mean[w] = m2[w] = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (i < pixels) {
#pragma unroll
            for (int v = 0; v < V; ++v) mean[v * W / V] += x[i].get(v);
        }
#pragma unroll
    for (int w = 0; w < W; ++w) mean[w] *= inv;
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (i < pixels) {
            x[i].pin();
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float d = x[i].get(v) - mean[v * W / V];
                m2[v * W / V] += d * d;
            }
        }
    float count = s.count;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        count = s.count;
        join_spread(s.mean[w], s.m2[w], count, mean[w], m2[w], k);
    }
    s.count = count;
}

// .. that join_chunk needs for W sets a thread: a count for each row of them comes behind.
__host__ __device__ constexpr int join_floats2(int threads, int W, int rpar) { return sum_floats2(threads, W, rpar) + (threads + 1) / 2; }

// Joins the threads' sets to one for each group of the tile, in an order that the shape of the launch fixes: done(group, mean, squares) in
// one thread each.
template <int V, int W, typename F> __device__ __forceinline__ void join_chunk(const NormArgs &a, const Tile &t, Spread<W> &mine, float2 *lds, F done)
{
    const int nch = t.cols * W, threads = blockDim.x, per = a.D * W / V;
    float2 *second = lds + threads * W;
    float *counts = (float *)(lds + sum_floats2(threads, W, t.rpar));
    const float2 *sets = lds;
    int parts;
    if (64 % t.cols == 0 && t.rpar * t.cols == threads) { // lanes of a wavefront `cols` apart hold the same channels
        for (int o = 32; o >= t.cols; o /= 2) {
            const float cb = __shfl_down(mine.count, o);
            float count = mine.count;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float mb = __shfl_down(mine.mean[w], o), qb = __shfl_down(mine.m2[w], o);
                count = mine.count;
                join_spread(mine.mean[w], mine.m2[w], count, mb, qb, cb);
            }
            mine.count = count;
        }
        const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
        parts = threads / 64;
        if (lane < t.cols) {
#pragma unroll
            for (int w = 0; w < W; ++w) lds[wave * nch + lane * W + w] = make_float2(mine.mean[w], mine.m2[w]);
        }
        if (lane == 0) counts[wave] = mine.count; // (all pieces across have as many pixels)
        __syncthreads();
    } else {
        if (t.r < t.rpar) {
#pragma unroll
            for (int w = 0; w < W; ++w) lds[t.r * nch + t.col * W + w] = make_float2(mine.mean[w], mine.m2[w]);
        }
        parts = min(t.rpar, max(1, threads / nch));
        for (int q = threadIdx.x; q < parts; q += threads) {
            int n = 0;
#pragma unroll 1
            for (int r = q; r < t.rpar; r += parts) n += pixels_at(t, r);
            counts[q] = (float)(n * (V / W));
        }
        __syncthreads();
        if (parts < t.rpar) {
#pragma unroll 1
            for (int j = threadIdx.x; j < parts * nch; j += threads) {
                const int ch = j % nch;
                float mean = 0.f, m2 = 0.f, count = 0.f;
#pragma unroll 1
                for (int r = j / nch; r < t.rpar; r += parts) {
                    const float2 b = lds[r * nch + ch];
                    join_spread(mean, m2, count, b.x, b.y, (float)(pixels_at(t, r) * (V / W)));
                }
                second[j] = make_float2(mean, m2);
            }
            sets = second;
            __syncthreads();
        }
    }
    const int lane = threadIdx.x % kLanes, clusters = threads / kLanes;
    for (int g = threadIdx.x / kLanes; g < t.groups; g += clusters) {
        float mean = 0.f, m2 = 0.f, count = 0.f;
#pragma unroll 1
        for (int j = lane; j < parts * per; j += kLanes) {
            const int q = j / per, i = j - q * per;
            const float2 b = sets[q * nch + g * per + i];
            join_spread(mean, m2, count, b.x, b.y, counts[q]);
        }
        for (int o = kLanes / 2; o; o /= 2) {
            const float mb = __shfl_down(mean, o, kLanes), qb = __shfl_down(m2, o, kLanes), cb = __shfl_down(count, o, kLanes);
            join_spread(mean, m2, count, mb, qb, cb);
        }
        if (lane == 0) done(g, mean, m2);
    }
}

// mean, rstd of group g of the tile, which one thread hands to the others and, of an image's first chunk, to the caller.
__device__ __forceinline__ void keep_stats(const NormArgs &a, const Tile &t, int g, float mean, float m2, float *stats)
{
    const float rstd = 1.f / sqrtf(m2 / ((float)a.P * (float)a.D) + a.eps);
    stats[2 * g] = mean;
    stats[2 * g + 1] = rstd;
    if (t.s == 0 && a.mean) {
        a.mean[t.n * a.G + t.g0 + g] = mean;
        a.rstd[t.n * a.G + t.g0 + g] = rstd;
    }
}

// ACT: a qrm_act, or kAnyAct: the call's, looked up value by value (narrow pieces).
constexpr int kAnyAct = -1;
template <int ACT> __device__ __forceinline__ float activate(float z)
{
    if (ACT == QRM_ACT_RELU) return z < 0.f ? 0.f : z; // (a NaN stays one)
    if (ACT == QRM_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f)); // both within 1 ulp
    return z;
}

// A ReLU's argument, rounded product by product, as the definition is written, forward and backward alike: where y is above zero its slope is one.
__device__ __forceinline__ float relu_z(float d, float rstd, float gamma, float beta)
{
#pragma clang fp contract(off)
    return (d * rstd) * gamma + beta;
}

// act(gamma (x - mean) rstd + beta) of one thread's channels.  gamma and beta are read before anything is waited for.
template <int V, int W> struct Affine {
    float mean[W], rstd[W], gamma[V], scale[V], bias[V]; // scale: gamma rstd
    int group[W];
    __device__ __forceinline__ Affine(const NormArgs &a, const Tile &t)
    {
#pragma unroll
        for (int w = 0; w < W; ++w) group[w] = (t.col * V + w * (V / W)) / a.D;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = t.c0 + min(t.col, t.cols - 1) * V + v;
            gamma[v] = a.gamma ? a.gamma[c] : 1.f;
            bias[v] = a.beta ? a.beta[c] : 0.f;
        }
    }
    __device__ __forceinline__ void set(const float *stats)
    {
#pragma unroll
        for (int w = 0; w < W; ++w) {
            mean[w] = stats[2 * group[w]];
            rstd[w] = stats[2 * group[w] + 1];
#pragma unroll
            for (int v = 0; v < V / W; ++v) scale[w * (V / W) + v] = gamma[w * (V / W) + v] * rstd[w];
        }
    }
    template <int KIND> __device__ __forceinline__ float value(int v, float d) const
    {
        return activate<KIND>(KIND == QRM_ACT_RELU ? relu_z(d, rstd[v * W / V], gamma[v], bias[v]) : fmaf(d, scale[v], bias[v]));
    }
    template <int ACT, typename T> __device__ __forceinline__ Words<T, V> apply(const Words<T, V> &x, int act) const
    {
        float f[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float d = x.get(v) - mean[v * W / V];
            if constexpr (ACT != kAnyAct) f[v] = value<ACT>(v, d);
            else f[v] = act == QRM_ACT_SILU ? value<QRM_ACT_SILU>(v, d) : act == QRM_ACT_RELU ? value<QRM_ACT_RELU>(v, d) : value<QRM_ACT_NONE>(v, d);
        }
        Words<T, V> y;
        y.set(f);
        return y;
    }
};

// One launch: R pixels a thread, a whole tile a workgroup.  1 image of 256 pixels and 512 channels (bf16, silu) 6.3 us, of which 4 are launch and
// the first loads; two launches 9.7.
template <typename T, int V, int W, int ACT, int R, bool STREAM> __global__ __launch_bounds__(kMaxThreads) void norm_whole_kernel(NormArgs a)
{
    extern __shared__ __align__(16) float2 lds[];
    float *stats = (float *)(lds + join_floats2(blockDim.x, W, a.rpar)); // mean, rstd of the tile's groups
    const Tile t = find_tile<V>(a);
    const bool active = t.r < t.rpar;
    const int pixels = active ? pixels_at(t, t.r) : 0;
    Words<T, V> x[R];
    if (active) read_chunk<T, V, R>(x_at<T, V>(a, t, 0), t.step * a.xp, t.r, pixels, a.xp, x);
    Affine<V, W> f(a, t);
    Spread<W> mine;
#pragma unroll
    for (int w = 0; w < W; ++w) mine.mean[w] = mine.m2[w] = 0.f;
    mine.count = 0.f;
    spread_batch<T, V, W, R>(mine, x, pixels);
    join_chunk<V, W>(a, t, mine, lds, [&](int g, float mean, float m2) { keep_stats(a, t, g, mean, m2, stats); });
    __syncthreads();
    if (!active) return;
    f.set(stats);
    T *q = (T *)a.y + y_offset<V>(a, t, t.r);
    const int64_t ys = t.step * a.yp;
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (i < pixels) {
            x[i].pin();
            store_words<STREAM, T, V>(q + i * ys, f.template apply<ACT>(x[i], a.act));
        }
}

// Two launches, the first: (mean, squares) of every group of the tile over this chunk.  67 MB in 15.6 us, 4.3 TB/s.
template <typename T, int V, int W> __global__ __launch_bounds__(kMaxThreads) void norm_stats_kernel(NormArgs a)
{
    constexpr int R = 8;
    extern __shared__ __align__(16) float2 lds[];
    const Tile t = find_tile<V>(a);
    Spread<W> mine;
#pragma unroll
    for (int w = 0; w < W; ++w) mine.mean[w] = mine.m2[w] = 0.f;
    mine.count = 0.f;
    if (t.r < t.rpar) {
        const int pixels = pixels_at(t, t.r);
        const T *p = x_at<T, V>(a, t, pixels ? t.r : 0);
        const int64_t step = t.step * a.xp;
        Words<T, V> x[R], next[R]; // the next pixels are on their way while these are added
        fetch<T, V, R, false>(p, step, 0, pixels, x);
        for (int at = 0; at < pixels; at += R) {
            if (at + R < pixels) fetch<T, V, R, false>(p, step, at + R, pixels, next);
            spread_batch<T, V, W, R>(mine, x, pixels - at);
#pragma unroll
            for (int i = 0; i < R; ++i) x[i] = next[i];
        }
    }
    join_chunk<V, W>(a, t, mine, lds, [&](int g, float mean, float m2) { *part_at(a, t, g, t.s) = make_float2(mean, m2); });
}

// .. the second: joins the chunks' parts and writes the outputs.  134 MB in 22.5 us, 6.0 TB/s.
template <typename T, int V, int W, int ACT, bool STREAM> __global__ __launch_bounds__(kMaxThreads) void norm_apply_kernel(NormArgs a)
{
    constexpr int R = 4;
    extern __shared__ __align__(16) float2 lds[]; // mean, rstd of the tile's groups
    float *stats = (float *)lds;
    const Tile t = find_tile<V>(a);
    const int lanes = lanes_for(t.groups), lane = threadIdx.x & (lanes - 1), first = threadIdx.x / lanes;
    Parts parts(part_at(a, t, min(first, t.groups - 1), 0), a.parts, lane, lanes);
    // from the last pixels on, which the first launch has read last and the caches may still hold; the first of them are on their way while the
    // parts are joined
    int left = t.r < t.rpar ? pixels_at(t, t.r) : 0;
    const T *p = x_at<T, V>(a, t, left ? t.r : 0);
    const int64_t xs = t.step * a.xp, ys = t.step * a.yp;
    Words<T, V> x[R], next[R];
    if (t.r < t.rpar) fetch<T, V, R, true>(p, xs, left, left, x);
    Affine<V, W> f(a, t);
    for (int g = first; g < t.groups; g += blockDim.x / lanes) {
        if (g != first) parts = Parts(part_at(a, t, g, 0), a.parts, lane, lanes);
        float mean = 0.f, m2 = 0.f, count = 0.f;
        // pixels of chunk s: its share of every round, and what the last round leaves for it
        const int64_t round = (int64_t)a.parts * a.parts_rpar;
        const float share = (float)(a.P / round) * a.parts_rpar;
        const int rest = (int)(a.P % round);
        parts.each([&](float2 v, int s) {
            join_spread(mean, m2, count, v.x, v.y, (share + (float)max(0, min(a.parts_rpar, rest - s * a.parts_rpar))) * (float)a.D);
        });
        for (int o = lanes / 2; o; o /= 2) {
            const float mb = __shfl_down(mean, o, lanes), qb = __shfl_down(m2, o, lanes), cb = __shfl_down(count, o, lanes);
            join_spread(mean, m2, count, mb, qb, cb);
        }
        if (lane == 0) keep_stats(a, t, g, mean, m2, stats);
    }
    __syncthreads();
    if (!left) return;
    f.set(stats);
    T *q = (T *)a.y + y_offset<V>(a, t, t.r);
    for (; left > 0; left -= R) {
        if (left > R) fetch<T, V, R, true>(p, xs, left - R, left, next);
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < left) store_words<STREAM, T, V>(q + (left - 1 - i) * ys, f.template apply<ACT>(x[i], a.act));
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = next[i];
    }
}

// ---------------------------------------------------------------- backward

// What a thread keeps of its channels.  d = x - mean throughout; h = d rstd.
template <int V, int W, int ACT> struct Slopes {
    float mean[W], rstd[W], gamma[V], beta[V];
    __device__ __forceinline__ Slopes(const NormArgs &a, const Tile &t)
    {
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const int64_t g = t.n * a.G + (t.c0 + t.col * V + w * (V / W)) / a.D;
            mean[w] = a.mean[g];
            rstd[w] = a.rstd[g];
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = t.c0 + t.col * V + v;
            gamma[v] = a.gamma ? a.gamma[c] : 1.f;
            beta[v] = a.beta ? a.beta[c] : 0.f;
        }
    }
    // dy act'(z)
    template <int KIND> __device__ __forceinline__ float dz_of(int v, float d, float dy) const
    {
#pragma clang fp contract(off)
        const float r = rstd[v * W / V];
        if (KIND == QRM_ACT_NONE) return dy;
        if (KIND == QRM_ACT_RELU) return relu_z(d, r, gamma[v], beta[v]) <= 0.f ? 0.f : dy;
        const float z = fmaf(d, gamma[v] * r, beta[v]); // (gamma rstd is the same for all pixels: kept in a register)
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f));
        return dy * (s * fmaf(z, 1.f - s, 1.f));
    }
    __device__ __forceinline__ float dz(int v, float d, float dy, int act) const
    {
        if (ACT != kAnyAct) return dz_of<ACT>(v, d, dy);
        return act == QRM_ACT_SILU ? dz_of<QRM_ACT_SILU>(v, d, dy) : act == QRM_ACT_RELU ? dz_of<QRM_ACT_RELU>(v, d, dy) : dy;
    }
};

// dx = rstd (gamma dz - A - h B) = dz k1 - (d k3 + k2).  A group of one value has no gradient: its factors are zeros, not what rounding
// leaves of a difference.
template <int V, int W> struct InputGrad {
    float k2[W], k3[W], k1[V];
    template <int ACT> __device__ __forceinline__ InputGrad(const NormArgs &a, const Tile &t, const Slopes<V, W, ACT> &c, const float *sums)
    {
        const float some = a.P * a.D > 1 ? 1.f : 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const int g = (t.col * V + w * (V / W)) / a.D;
            const float r = c.rstd[w] * some;
            k2[w] = r * sums[2 * g];
            k3[w] = r * c.rstd[w] * sums[2 * g + 1];
        }
#pragma unroll
        for (int v = 0; v < V; ++v) k1[v] = c.gamma[v] * c.rstd[v * W / V] * some;
    }
    __device__ __forceinline__ float dx(int v, float d, float dz) const { return fmaf(dz, k1[v], -fmaf(d, k3[v * W / V], k2[v * W / V])); }
};

// Sums (sum dz, sum dz d) over the threads: by_channel(channel of the tile, sum dz, sum dz h) and by_group(group, both weighted with gamma) in one
// thread each, all channels before the first group.
template <int V, int W, int ACT, typename FC, typename FG>
__device__ __forceinline__ void sum_chunk(const NormArgs &a, const Tile &t, const Slopes<V, W, ACT> &c, const float (&b)[V], const float (&g)[V], float2 *lds, FC by_channel, FG by_group)
{
    const int nch = t.cols * V, threads = blockDim.x;
    if (t.r < t.rpar) {
#pragma unroll
        for (int v = 0; v < V; ++v) lds[t.r * nch + t.col * V + v] = make_float2(b[v], g[v] * c.rstd[v * W / V]);
    }
    __syncthreads();
    const int parts = min(t.rpar, max(1, threads / nch));
    float2 *second = lds + threads * V;
    const float2 *sums = lds;
    if (parts < t.rpar) {
#pragma unroll 1
        for (int j = threadIdx.x; j < parts * nch; j += threads) {
            const int ch = j % nch;
            float2 s = make_float2(0.f, 0.f);
#pragma unroll 2
            for (int r = j / nch; r < t.rpar; r += parts) {
                s.x += lds[r * nch + ch].x;
                s.y += lds[r * nch + ch].y;
            }
            second[j] = s;
        }
        sums = second;
        __syncthreads();
    }
    // the channels' totals, in place of what is not read, or of what the same thread reads (one pixel at a time)
    float2 *total = parts < t.rpar || t.rpar == 1 ? lds : second;
#pragma unroll 1
    for (int j = threadIdx.x; j < nch; j += threads) {
        double sb = 0.0, sg = 0.0; // (few channels have many parts)
#pragma unroll 2
        for (int q = 0; q < parts; ++q) {
            sb += sums[q * nch + j].x;
            sg += sums[q * nch + j].y;
        }
        const float2 s = make_float2((float)sb, (float)sg);
        by_channel(j, s.x, s.y);
        const float w = a.gamma ? a.gamma[t.c0 + j] : 1.f;
        total[j] = make_float2(s.x * w, s.y * w);
    }
    __syncthreads();
    const int lane = threadIdx.x % kLanes;
    for (int k = threadIdx.x / kLanes; k < t.groups; k += threads / kLanes) {
        float2 s = make_float2(0.f, 0.f);
#pragma unroll 1
        for (int i = lane; i < a.D; i += kLanes) {
            const float2 v = total[k * a.D + i];
            s.x += v.x;
            s.y += v.y;
        }
        for (int o = kLanes / 2; o; o /= 2) {
            s.x += __shfl_down(s.x, o, kLanes);
            s.y += __shfl_down(s.y, o, kLanes);
        }
        if (lane == 0) by_group(k, s.x, s.y);
    }
}

// dgamma, dbeta of up to 16 channels from c0 on: `terms` sums of each, added in a fixed order by a workgroup, in 64 bits: they may cancel, and are few.
// lds: blockDim.x / 2 float2s.
__device__ __forceinline__ void channel_grads(const NormArgs &a, int64_t terms, int c0, float2 *lds)
{
    const int c = c0 + threadIdx.x % 16, r = threadIdx.x / 16, rows = blockDim.x / 16;
    double b = 0.0, g = 0.0;
    if (c < a.C) {
#pragma unroll 8
        for (int64_t k = r; k < terms; k += rows) {
            const float2 v = a.chan[k * a.C + c];
            b += v.x;
            g += v.y;
        }
    }
    // lanes 16 apart hold the same channel
    for (int o = 32; o >= 16; o /= 2) {
        b += __shfl_down(b, o);
        g += __shfl_down(g, o);
    }
    double2 *sums = (double2 *)lds;
    if ((threadIdx.x & 63) < 16) sums[threadIdx.x / 64 * 16 + threadIdx.x % 16] = make_double2(b, g);
    __syncthreads();
    if (threadIdx.x < 16 && c < a.C) {
        for (int k = 1; k < (int)blockDim.x / 64; ++k) {
            b += sums[k * 16 + threadIdx.x].x;
            g += sums[k * 16 + threadIdx.x].y;
        }
        if (a.dbeta) a.dbeta[c] = (float)b;
        if (a.dgamma) a.dgamma[c] = (float)g;
    }
}
__global__ __launch_bounds__(kThreads) void norm_channels_kernel(NormArgs a)
{
    __shared__ __align__(16) float2 lds[kThreads / 2];
    channel_grads(a, a.N * a.parts, blockIdx.x * 16, lds);
}

// One launch (and one for the channels of several images): R pixels a thread, a whole tile a workgroup.  dz stays in registers beside the
// input.  1 image of 256 pixels and 512 channels 7.3 us, two launches 11.6.
template <typename T, int V, int W, int ACT, int R> __global__ __launch_bounds__(kMaxThreads / 2) void norm_grad_whole_kernel(NormArgs a)
{
    extern __shared__ __align__(16) float2 lds[];
    float *sums = (float *)(lds + sum_floats2(blockDim.x, V, a.rpar)); // A, B of the tile's groups
    const Tile t = find_tile<V>(a);
    const int64_t xs = t.step * a.xp, ys = t.step * a.yp;
    const bool active = t.r < t.rpar;
    const float inv = 1.f / ((float)a.P * (float)a.D);
    const int pixels = active ? pixels_at(t, t.r) : 0;
    const Slopes<V, W, ACT> c(a, t);
    Words<T, V> x[R];
    float dz[R][V], b[V], g[V];
#pragma unroll
    for (int v = 0; v < V; ++v) b[v] = g[v] = 0.f;
    if (active) {
        Words<T, V> dy[R];
        read_chunk<T, V, R>(x_at<T, V>(a, t, 0), xs, t.r, pixels, a.xp, x);
        read_chunk<T, V, R>((const T *)a.dy + y_offset<V>(a, t, 0), ys, t.r, pixels, a.yp, dy);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (i >= pixels) dy[i] = Words<T, V>{};
#pragma unroll
            for (int v = 0; v < V; ++v) {
                // (no pixel: no gradient; its x is another one's of the channel)
                const float d = x[i].get(v) - c.mean[v * W / V];
                dz[i][v] = c.dz(v, d, dy[i].get(v), a.act);
                b[v] += dz[i][v];
                g[v] += dz[i][v] * d;
            }
        }
    }
    sum_chunk(a, t, c, b, g, lds, [&](int ch, float sb, float sg) {
        if (a.N > 1) {
            if (a.chan) a.chan[t.n * a.C + t.c0 + ch] = make_float2(sb, sg);
        } else {
            if (a.dbeta) a.dbeta[t.c0 + ch] = sb;
            if (a.dgamma) a.dgamma[t.c0 + ch] = sg;
        }
    }, [&](int k, float sa, float sb) { sums[2 * k] = sa * inv, sums[2 * k + 1] = sb * inv; });
    __syncthreads();
    if (!active || !a.dx) return;
    const InputGrad<V, W> f(a, t, c, sums);
    T *q = (T *)a.dx + (x_at<T, V>(a, t, t.r) - (const T *)a.x);
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (i < pixels) {
            float d[V];
            x[i].pin();
#pragma unroll
            for (int v = 0; v < V; ++v) d[v] = f.dx(v, x[i].get(v) - c.mean[v * W / V], dz[i][v]);
            Words<T, V> out;
            out.set(d);
            store_words<false, T, V>(q + i * xs, out);
        }
}

// Two launches, the first: sums of dz and dz h over the chunk, channel by channel and weighted with gamma group by group.  134 MB in 30.3 us, 4.4
// TB/s, and 17 us of arithmetic, not all of it beside the loads.  A thread adds runs of kRun pixels, then their sums, of which kNormRow pixels leave 43: with
// thousands of equal numbers one after the other, roundings that all go one way would grow to a thousand units in the last place.
constexpr int kRun = 48;
template <typename T, int V, int W, int ACT> __global__ __launch_bounds__(kMaxThreads) void norm_grad_sums_kernel(NormArgs a)
{
    constexpr int R = 3;
    extern __shared__ __align__(16) float2 lds[];
    const Tile t = find_tile<V>(a);
    const int pixels = t.r < t.rpar ? pixels_at(t, t.r) : 0;
    const T *p = x_at<T, V>(a, t, pixels ? t.r : 0);
    const T *q = (const T *)a.dy + y_offset<V>(a, t, pixels ? t.r : 0);
    const int64_t xs = t.step * a.xp, ys = t.step * a.yp;
    Words<T, V> x[R], dy[R], next_x[R], next_dy[R]; // the next pixels are on their way while these are added
    if (t.r < t.rpar) {
        fetch<T, V, R, false>(p, xs, 0, pixels, x);
        fetch<T, V, R, false>(q, ys, 0, pixels, dy);
    }
    const Slopes<V, W, ACT> c(a, t);
    float2 *runs = lds + threadIdx.x * V; // the thread's sums of the runs so far
    float b[V], g[V];
#pragma unroll
    for (int v = 0; v < V; ++v) b[v] = g[v] = 0.f;
    for (int at = 0; at < pixels; at += R) {
        if (at + R < pixels) {
            fetch<T, V, R, false>(p, xs, at + R, pixels, next_x);
            fetch<T, V, R, false>(q, ys, at + R, pixels, next_dy);
        }
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (at + i < pixels) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float d = x[i].get(v) - c.mean[v * W / V], z = c.dz(v, d, dy[i].get(v), a.act);
                    b[v] += z;
                    g[v] += z * d;
                }
            }
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = next_x[i], dy[i] = next_dy[i];
        if ((at / R + 1) % (kRun / R) == 0 || at + R >= pixels) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (at >= kRun) b[v] += runs[v].x, g[v] += runs[v].y;
                if (at + R < pixels) runs[v] = make_float2(b[v], g[v]), b[v] = g[v] = 0.f;
            }
        }
    }
    sum_chunk(a, t, c, b, g, lds, [&](int ch, float sb, float sg) {
        if (a.chan) a.chan[((size_t)t.n * a.parts + t.s) * a.C + t.c0 + ch] = make_float2(sb, sg);
    },
              [&](int k, float sa, float sb) { *part_at(a, t, k, t.s) = make_float2(sa, sb); });
}

// .. the second: dx, and in the workgroups behind those dgamma and dbeta of 16 channels each.  201 MB in 32.3 us, 6.2 TB/s.
template <typename T, int V, int W, int ACT, bool STREAM> __global__ __launch_bounds__(kMaxThreads) void norm_grad_apply_kernel(NormArgs a, uint32_t apply_blocks)
{
    constexpr int R = 2;
    extern __shared__ __align__(16) float2 lds[];
    if (blockIdx.x >= apply_blocks) {
        channel_grads(a, a.N * a.parts, (blockIdx.x - apply_blocks) * 16, lds);
        return;
    }
    float *sums = (float *)lds;
    const Tile t = find_tile<V>(a);
    const int lanes = lanes_for(t.groups), lane = threadIdx.x & (lanes - 1), first = threadIdx.x / lanes;
    Parts parts(part_at(a, t, min(first, t.groups - 1), 0), a.parts, lane, lanes);
    int left = t.r < t.rpar ? pixels_at(t, t.r) : 0; // (from the last pixels on, as above)
    const T *p = x_at<T, V>(a, t, left ? t.r : 0);
    const T *q = (const T *)a.dy + y_offset<V>(a, t, left ? t.r : 0);
    const int64_t xs = t.step * a.xp, ys = t.step * a.yp;
    Words<T, V> x[R], dy[R], next_x[R], next_dy[R];
    if (t.r < t.rpar) {
        fetch<T, V, R, true>(p, xs, left, left, x);
        fetch<T, V, R, true>(q, ys, left, left, dy);
    }
    const Slopes<V, W, ACT> c(a, t);
    const float inv = 1.f / ((float)a.P * (float)a.D);
    for (int k = first; k < t.groups; k += blockDim.x / lanes) {
        if (k != first) parts = Parts(part_at(a, t, k, 0), a.parts, lane, lanes);
        float2 v = make_float2(0.f, 0.f);
        parts.each([&](float2 p, int) {
            v.x += p.x;
            v.y += p.y;
        });
        for (int o = lanes / 2; o; o /= 2) {
            v.x += __shfl_down(v.x, o, lanes);
            v.y += __shfl_down(v.y, o, lanes);
        }
        if (lane == 0) sums[2 * k] = v.x * inv, sums[2 * k + 1] = v.y * inv;
    }
    __syncthreads();
    if (!left) return;
    const InputGrad<V, W> f(a, t, c, sums);
    T *w = (T *)a.dx + (p - (const T *)a.x);
    for (; left > 0; left -= R) {
        if (left > R) {
            fetch<T, V, R, true>(p, xs, left - R, left, next_x);
            fetch<T, V, R, true>(q, ys, left - R, left, next_dy);
        }
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < left) {
                float out[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float d = x[i].get(v) - c.mean[v * W / V];
                    out[v] = f.dx(v, d, c.dz(v, d, dy[i].get(v), a.act));
                }
                Words<T, V> r;
                r.set(out);
                store_words<STREAM, T, V>(w + (left - 1 - i) * xs, r);
            }
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = next_x[i], dy[i] = next_dy[i];
    }
}

NormArgs norm_args(const NormCall &c, const NormPlan &p, const NormCut &cut, void *ws)
{
    NormArgs a{};
    a.x = c.x; a.dy = c.dy; a.y = c.y; a.dx = c.dx;
    a.gamma = c.gamma; a.beta = c.beta;
    a.mean = c.mean; a.rstd = c.rstd; a.dgamma = c.dgamma; a.dbeta = c.dbeta;
    a.N = c.d.N; a.P = c.d.P;
    a.xp = c.d.x_pixel; a.xn = c.d.x_image; a.yp = c.d.y_pixel; a.yn = c.d.y_image;
    a.C = c.d.C; a.G = c.d.groups; a.D = c.d.C / c.d.groups;
    a.ct = cut.ct; a.tiles = cut.tiles; a.chunks = cut.chunks; a.rpar = cut.threads / (cut.ct / p.V);
    a.side = p.whole ? std::max(1, 128 / (cut.ct * type_bytes(c.d.type))) : 1;
    a.turned = a.side > 1 ? cut.blocks(a.N) / (kDies * a.side) * (kDies * a.side) : 0;
    a.parts = p.first.chunks; a.parts_rpar = p.first.threads / (p.first.ct / p.V);
    a.eps = c.d.eps;
    a.act = c.d.act;
    a.part = (float2 *)ws;
    a.chan = p.channels ? a.part + p.part_words : nullptr;
    return a;
}

// f(V, W, activation) as constants.
template <int V, typename F> hipError_t with_sets(int W, int act, F &&f)
{
    auto with_act = [&](auto sets) {
        std::integral_constant<int, V> width;
        if constexpr (V < 4) return f(width, sets, std::integral_constant<int, kAnyAct>());
        else return act == QRM_ACT_SILU ? f(width, sets, std::integral_constant<int, QRM_ACT_SILU>())
                    : act == QRM_ACT_RELU ? f(width, sets, std::integral_constant<int, QRM_ACT_RELU>()) : f(width, sets, std::integral_constant<int, QRM_ACT_NONE>());
    };
    if constexpr (V == 8) {
        if (W == 8) return with_act(std::integral_constant<int, 8>());
    }
    if constexpr (V >= 4) {
        if (W == 4) return with_act(std::integral_constant<int, 4>());
    }
    if constexpr (V >= 2) {
        if (W == 2) return with_act(std::integral_constant<int, 2>());
    }
    return with_act(std::integral_constant<int, 1>());
}
template <typename T, typename F> hipError_t with_width(const NormPlan &p, int act, F &&f)
{
    if constexpr (sizeof(T) == 2) {
        if (p.V == 8) return with_sets<8>(p.W, act, f);
    }
    return p.V == 4 ? with_sets<4>(p.W, act, f) : p.V == 2 ? with_sets<2>(p.W, act, f) : with_sets<1>(p.W, act, f);
}

template <typename T> hipError_t norm_forward(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s)
{
    const NormArgs a = norm_args(c, p, p.first, ws);
    const dim3 grid(p.first.blocks(c.d.N)), block(p.first.threads);
    return with_width<T>(p, c.d.act, [&](auto width, auto sets, auto act) {
        constexpr int V = decltype(width)::value, W = decltype(sets)::value, ACT = decltype(act)::value;
        const size_t join = join_floats2(p.first.threads, W, a.rpar) * sizeof(float2);
        if (p.whole) {
            const size_t own = 2 * (p.first.ct / a.D) * sizeof(float);
            auto whole = [&](auto stream) {
                constexpr bool STREAM = decltype(stream)::value;
                if (p.pixels > kNormFew) hipLaunchKernelGGL((norm_whole_kernel<T, V, W, ACT, norm_many(false, W), STREAM>), grid, block, join + own, s, a);
                else hipLaunchKernelGGL((norm_whole_kernel<T, V, W, ACT, kNormFew, STREAM>), grid, block, join + own, s, a);
            };
            p.stream ? whole(std::true_type()) : whole(std::false_type());
            return hipGetLastError();
        }
        hipLaunchKernelGGL((norm_stats_kernel<T, V, W>), grid, block, join, s, a);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        auto apply = [&](auto stream) {
            hipLaunchKernelGGL((norm_apply_kernel<T, V, W, ACT, decltype(stream)::value>), dim3(p.second.blocks(c.d.N)), dim3(p.second.threads),
                               2 * (p.second.ct / a.D) * sizeof(float), s, norm_args(c, p, p.second, ws));
        };
        p.stream ? apply(std::true_type()) : apply(std::false_type());
        return hipGetLastError();
    });
}

template <typename T> hipError_t norm_backward(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s)
{
    const NormArgs a = norm_args(c, p, p.first, ws);
    const uint32_t extra = p.channels ? (c.d.C + 15) / 16 : 0;
    const dim3 grid(p.first.blocks(c.d.N)), block(p.first.threads);
    return with_width<T>(p, c.d.act, [&](auto width, auto sets, auto act) {
        constexpr int V = decltype(width)::value, W = decltype(sets)::value, ACT = decltype(act)::value;
        const size_t sum = sum_floats2(p.first.threads, V, a.rpar) * sizeof(float2);
        if (p.whole) {
            const size_t own = 2 * (p.first.ct / a.D) * sizeof(float);
            if (p.pixels > kNormFew) hipLaunchKernelGGL((norm_grad_whole_kernel<T, V, W, ACT, norm_many(true, W)>), grid, block, sum + own, s, a);
            else hipLaunchKernelGGL((norm_grad_whole_kernel<T, V, W, ACT, kNormFew>), grid, block, sum + own, s, a);
            hipError_t e = hipGetLastError();
            if (e != hipSuccess || !extra) return e;
            hipLaunchKernelGGL(norm_channels_kernel, dim3(extra), dim3(kThreads), 0, s, a);
            return hipGetLastError();
        }
        hipLaunchKernelGGL((norm_grad_sums_kernel<T, V, W, ACT>), grid, block, sum, s, a);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        const uint32_t apply = c.dx ? p.second.blocks(c.d.N) : 0;
        const size_t own = std::max(2 * (p.second.ct / a.D) * sizeof(float), p.second.threads / 2 * sizeof(float2));
        auto launch = [&](auto stream) {
            hipLaunchKernelGGL((norm_grad_apply_kernel<T, V, W, ACT, decltype(stream)::value>), dim3(apply + extra), dim3(p.second.threads), own, s,
                               norm_args(c, p, p.second, ws), apply);
        };
        p.stream ? launch(std::true_type()) : launch(std::false_type());
        return hipGetLastError();
    });
}

} // namespace
} // namespace qrm
