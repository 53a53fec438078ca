// Group norm with an activation, channels last, forward and backward (qrm_group_norm, qrm_group_norm_backward).
//
// The work is cut into tiles of whole groups, at least a 128-byte line wide where the map is, and a tile's pixels into chunks, one to
// a workgroup.  A thread keeps one piece of V channels (up to 16 bytes) and walks down the chunk's pixels, so that scale, bias and
// statistics of its channels stay in registers.  Statistics need all of a group before the first output: a first launch leaves each chunk's
// part, a second one joins the parts of its tile in a fixed order and applies them.  Bound by memory: the formulas are 12 (backward:
// 25) operations for 4 (6) bytes of a 16-bit type.
#include "qrm_train.h"

#include <algorithm>
#include <numeric>
#include <type_traits>

namespace qrm {
namespace {

constexpr int kMaxThreads = 1024;
// Floats that column_sums needs for W sums a thread.  Workgroups of more than 256 threads are those of groups wider than 256 pieces:
// one group a tile and one pixel at a time, so there are no sums over pixels side by side.
__host__ __device__ constexpr int sum_floats(int threads, int W) { return (threads > 256 ? 1 : 2) * threads * W; }

struct NormArgs {
    const void *x, *dy;
    void *y, *dx;
    const float *gamma, *beta;
    float *mean, *rstd, *dgamma, *dbeta;
    float2 *part;          // [N][tiles][chunks][groups of a tile]: (mean, sum of squares about it), backward (sum gamma dz, sum gamma dz h)
    float2 *chan;          // backward: [N * chunks][C]: (sum dz, sum dz h)
    int64_t N, P, rows;
    int64_t xp, xn, yp, yn;
    int C, G, D, ct, tiles, chunks;
    float eps;
};

// What a workgroup is about: its image, channels and pixels, and its threads' places in them.
struct Tile {
    int64_t n, row0, rows; // image, first pixel, pixels
    int t, s;              // tile, chunk
    int c0, g0, groups;    // first channel and group, number of groups
    int cols, rpar;        // pieces across, pixels side by side
    int r, col;            // this thread's; r >= rpar: none
};

template <int V> __device__ __forceinline__ Tile find_tile(const NormArgs &a)
{
    Tile t;
    uint32_t b = blockIdx.x;
    t.t = b % a.tiles;
    b /= a.tiles;
    t.s = b % a.chunks;
    t.n = b / a.chunks;
    t.c0 = t.t * a.ct;
    const int cw = min(a.ct, a.C - t.c0);
    t.g0 = t.c0 / a.D;
    t.groups = cw / a.D;
    t.cols = cw / V;
    t.rpar = blockDim.x / t.cols;
    t.r = threadIdx.x / t.cols;
    t.col = threadIdx.x % t.cols;
    t.row0 = t.s * a.rows;
    t.rows = min(a.rows, a.P - t.row0);
    return t;
}

// Sums over the pixels side by side: w[0..W) of each thread -> *sums, sums over r for `nch` = cols * W columns, in `parts` rows that
// are still to be added.  The order is fixed by the launch's shape.  lds: sum_floats(threads, W) floats.
template <int W> __device__ __forceinline__ const float *column_sums(const Tile &t, const float (&w)[W], float *lds, int *nch_out, int *parts_out)
{
    const int nch = t.cols * W, threads = blockDim.x;
    float *second = lds + threads * W;
    __syncthreads(); // (the last call's readers are done)
    if (t.r < t.rpar) {
#pragma unroll
        for (int i = 0; i < W; ++i) lds[t.r * nch + t.col * W + i] = w[i];
    }
    __syncthreads();
    *nch_out = nch;
    const int parts = min(t.rpar, max(1, threads / nch));
    *parts_out = parts;
    if (parts == t.rpar) return lds;
    for (int j = threadIdx.x; j < parts * nch; j += threads) {
        const int ch = j % nch;
        float s = 0.f;
        for (int r = j / nch; r < t.rpar; r += parts) s += lds[r * nch + ch];
        second[j] = s;
    }
    __syncthreads();
    return second;
}

constexpr int kLanes = 16; // lanes that join a group's columns

// The sum of a group's columns, each weighted with weight(column) -> out[group], for all groups of the tile.  `per` columns a group.
template <typename F> __device__ __forceinline__ void join_groups(const float *sums, int nch, int parts, int groups, int per, float *out, F weight)
{
    const int lane = threadIdx.x % kLanes, clusters = blockDim.x / kLanes;
    for (int g = threadIdx.x / kLanes; g < groups; g += clusters) {
        float s = 0.f;
        for (int q = 0; q < parts; ++q)
            for (int i = lane; i < per; i += kLanes) s += sums[q * nch + g * per + i] * weight(g * per + i);
        for (int o = kLanes / 2; o; o /= 2) s += __shfl_xor(s, o, kLanes);
        if (lane == 0) out[g] = s;
    }
}

// Sums w over the tile's pixels and every group's channels; each thread gets its channels' groups.
template <int V, bool UNI> __device__ __forceinline__ void group_sums(const NormArgs &a, const Tile &t, const float (&w)[UNI ? 1 : V], float (&out)[UNI ? 1 : V], float *lds, float *gsum)
{
    constexpr int W = UNI ? 1 : V;
    int nch, parts;
    const float *sums = column_sums<W>(t, w, lds, &nch, &parts);
    join_groups(sums, nch, parts, t.groups, UNI ? a.D / V : a.D, gsum, [](int) { return 1.f; });
    __syncthreads();
    if (t.r < t.rpar) {
#pragma unroll
        for (int i = 0; i < W; ++i) out[i] = gsum[(t.col * V + i) / a.D];
    }
}

template <typename T, int V> __device__ __forceinline__ const T *x_at(const NormArgs &a, const Tile &t)
{
    return (const T *)a.x + t.n * a.xn + (t.row0 + t.r) * a.xp + t.c0 + t.col * V;
}

// ---------------------------------------------------------------- forward

// A thread's mean and squares about it (Chan's update): values in batches of up to R pixels, whose own mean and squares are exact to
// rounding, joined one after the other.  Nothing cancels however far the mean lies from zero.
template <int W> struct Spread {
    float mean[W], m2[W];
    float count; // values behind each
};

template <typename T, int V, bool UNI, int R> __device__ __forceinline__ void spread_batch(Spread<UNI ? 1 : V> &s, const Pack<T, V> (&x)[R], int valid)
{
    constexpr int W = UNI ? 1 : V;
    const float k = (float)(valid * (V / W)), total = s.count + k, share = k / total;
    float sum[W];
#pragma unroll
    for (int w = 0; w < W; ++w) sum[w] = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) sum[UNI ? 0 : v] += i < valid ? (float)x[i].e[v] : 0.f;
    const float inv = 1.f / k;
    float m2[W], mb[W];
#pragma unroll
    for (int w = 0; w < W; ++w) { mb[w] = sum[w] * inv; m2[w] = 0.f; }
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float d = i < valid ? (float)x[i].e[v] - mb[UNI ? 0 : v] : 0.f;
            m2[UNI ? 0 : v] += d * d;
        }
    const float cross = s.count * share;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const float delta = mb[w] - s.mean[w];
        s.mean[w] += delta * share;
        s.m2[w] += m2[w] + delta * delta * cross;
    }
    s.count = total;
}

// First launch: (mean, squares) of every group of the tile over this chunk.
template <typename T, int V, bool UNI> __global__ __launch_bounds__(kMaxThreads) void norm_stats_kernel(NormArgs a)
{
    constexpr int W = UNI ? 1 : V, R = 8;
    extern __shared__ float lds[];
    const Tile t = find_tile<V>(a);
    float *gsum = lds + sum_floats(blockDim.x, W);
    Spread<W> s;
#pragma unroll
    for (int w = 0; w < W; ++w) s.mean[w] = s.m2[w] = 0.f;
    s.count = 0.f;
    if (t.r < t.rpar) {
        const T *p = x_at<T, V>(a, t);
        const int64_t step = t.rpar * a.xp;
        int64_t left = (t.rows - t.r + t.rpar - 1) / t.rpar; // pixels of this thread
        for (; left >= R; left -= R) {
            Pack<T, V> x[R];
#pragma unroll
            for (int i = 0; i < R; ++i) x[i] = load_pack<T, V>(p + i * step);
            p += R * step;
            spread_batch<T, V, UNI, R>(s, x, R);
        }
        if (left > 0) {
            Pack<T, V> x[R];
#pragma unroll
            for (int i = 0; i < R; ++i) x[i] = load_pack<T, V>(p + (i < left ? i : 0) * step);
            spread_batch<T, V, UNI, R>(s, x, (int)left);
        }
    }
    // the group's mean is the weighted mean of the threads', its squares theirs plus the weighted squares of the means' distances
    float w[W], mean[W], m2[W];
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = s.count * s.mean[i];
    group_sums<V, UNI>(a, t, w, mean, lds, gsum);
    const float inv = 1.f / ((float)t.rows * (float)a.D);
    if (t.r < t.rpar) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            mean[i] *= inv;
            const float d = s.mean[i] - mean[i];
            w[i] = s.m2[i] + s.count * d * d;
        }
    }
    float2 *part = a.part + (((size_t)t.n * a.tiles + t.t) * a.chunks + t.s) * (a.ct / a.D);
    for (int g = threadIdx.x; g < t.groups; g += blockDim.x) part[g].x = gsum[g] * inv;
    group_sums<V, UNI>(a, t, w, m2, lds, gsum);
    for (int g = threadIdx.x; g < t.groups; g += blockDim.x) part[g].y = gsum[g];
}

// (mean, squares, count) of two sets joined.
__device__ __forceinline__ void join_spread(float &mean, float &m2, float &count, float mean_b, float m2_b, float count_b)
{
    const float total = count + count_b;
    if (total > 0.f) {
        const float delta = mean_b - mean, share = count_b / total;
        mean += delta * share;
        m2 += m2_b + delta * delta * (count * share);
        count = total;
    }
}

template <int ACT> __device__ __forceinline__ float activate(float z)
{
    if (ACT == QRM_ACT_RELU) return z < 0.f ? 0.f : z; // (a NaN stays one)
    if (ACT == QRM_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f)); // both within 1 ulp
    return z;
}

// Second launch: joins the chunks' parts and writes act(gamma (x - mean) rstd + beta).
template <typename T, int V, int ACT> __global__ __launch_bounds__(kMaxThreads) void norm_apply_kernel(NormArgs a)
{
    constexpr int R = 4;
    extern __shared__ float lds[]; // mean, rstd of the tile's groups
    const Tile t = find_tile<V>(a);
    const int gt = a.ct / a.D;
    const float2 *part = a.part + ((size_t)t.n * a.tiles + t.t) * a.chunks * gt;
    const int lane = threadIdx.x & 63, waves = blockDim.x / 64;
    for (int g = threadIdx.x / 64; g < t.groups; g += waves) {
        float mean = 0.f, m2 = 0.f, count = 0.f;
        for (int s = lane; s < a.chunks; s += 64) {
            const float2 v = part[(size_t)s * gt + g];
            join_spread(mean, m2, count, v.x, v.y, (float)min(a.rows, a.P - s * a.rows) * (float)a.D);
        }
        for (int o = 32; o; o /= 2) {
            const float mb = __shfl_xor(mean, o), qb = __shfl_xor(m2, o), cb = __shfl_xor(count, o);
            // both lanes join in the same order
            if (lane & o) {
                float m = mb, q = qb, c = cb;
                join_spread(m, q, c, mean, m2, count);
                mean = m, m2 = q, count = c;
            } else {
                join_spread(mean, m2, count, mb, qb, cb);
            }
        }
        if (lane == 0) {
            const float rstd = 1.f / sqrtf(m2 / count + a.eps);
            lds[2 * g] = mean;
            lds[2 * g + 1] = rstd;
            if (t.s == 0 && a.mean) {
                a.mean[t.n * a.G + t.g0 + g] = mean;
                a.rstd[t.n * a.G + t.g0 + g] = rstd;
            }
        }
    }
    __syncthreads();
    if (t.r >= t.rpar) return;
    float mean[V], scale[V], bias[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = t.col * V + v, g = c / a.D;
        mean[v] = lds[2 * g];
        scale[v] = lds[2 * g + 1] * (a.gamma ? a.gamma[t.c0 + c] : 1.f);
        bias[v] = a.beta ? a.beta[t.c0 + c] : 0.f;
    }
    const T *p = x_at<T, V>(a, t);
    T *q = (T *)a.y + t.n * a.yn + (t.row0 + t.r) * a.yp + t.c0 + t.col * V;
    const int64_t xs = t.rpar * a.xp, ys = t.rpar * a.yp;
    auto one = [&](const Pack<T, V> &x) {
        Pack<T, V> y;
#pragma unroll
        for (int v = 0; v < V; ++v) y.e[v] = (T)activate<ACT>(((float)x.e[v] - mean[v]) * scale[v] + bias[v]);
        return y;
    };
    int64_t left = (t.rows - t.r + t.rpar - 1) / t.rpar;
    for (; left >= R; left -= R) {
        Pack<T, V> x[R];
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = load_pack<T, V>(p + i * xs);
#pragma unroll
        for (int i = 0; i < R; ++i) store_pack<T, V>(q + i * ys, one(x[i]));
        p += R * xs;
        q += R * ys;
    }
    for (; left > 0; --left, p += xs, q += ys) store_pack<T, V>(q, one(load_pack<T, V>(p)));
}

// ---------------------------------------------------------------- backward

// The parts of a channel's gradient formula that a thread keeps.
struct Channel {
    float mean, rstd, gamma, beta;
};
// Products and sums are rounded one by one, as written, and only what says fmaf is fused: whether a ReLU passes depends on a sign alone, and
// both launches have to see the same dz for a sum over one value to cancel it.
template <int ACT> __device__ __forceinline__ void grad_parts(const Channel &c, float x, float dy, float &h, float &dz)
{
#pragma clang fp contract(off)
    h = (x - c.mean) * c.rstd;
    dz = dy;
    if (ACT == QRM_ACT_NONE) return;
    const float z = h * c.gamma + c.beta;
    if (ACT == QRM_ACT_RELU) dz = z <= 0.f ? 0.f : dy;
    if (ACT == QRM_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f));
        dz = dy * (s * fmaf(z, 1.f - s, 1.f));
    }
}
__device__ __forceinline__ float grad_input(const Channel &c, float h, float dz, float sum_a, float sum_b)
{
#pragma clang fp contract(off)
    const float a = c.gamma * dz - sum_a;
    return c.rstd * fmaf(-h, sum_b, a);
}

template <int V> __device__ __forceinline__ void load_channels(const NormArgs &a, const Tile &t, Channel (&c)[V])
{
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int ch = t.c0 + t.col * V + v, g = ch / a.D;
        c[v].mean = a.mean[t.n * a.G + g];
        c[v].rstd = a.rstd[t.n * a.G + g];
        c[v].gamma = a.gamma ? a.gamma[ch] : 1.f;
        c[v].beta = a.beta ? a.beta[ch] : 0.f;
    }
}

// First launch: sums of dz and dz h over the chunk, channel by channel and weighted with gamma group by group.
template <typename T, int V, int ACT> __global__ __launch_bounds__(kMaxThreads) void norm_grad_sums_kernel(NormArgs a)
{
    constexpr int R = 4;
    extern __shared__ float lds[];
    const Tile t = find_tile<V>(a);
    float *gsum = lds + sum_floats(blockDim.x, V);
    float b[V], g[V];
#pragma unroll
    for (int v = 0; v < V; ++v) b[v] = g[v] = 0.f;
    if (t.r < t.rpar) {
        Channel c[V];
        load_channels<V>(a, t, c);
        const T *p = x_at<T, V>(a, t);
        const T *q = (const T *)a.dy + t.n * a.yn + (t.row0 + t.r) * a.yp + t.c0 + t.col * V;
        const int64_t xs = t.rpar * a.xp, ys = t.rpar * a.yp;
        auto add = [&](const Pack<T, V> &x, const Pack<T, V> &dy) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float h, dz;
                grad_parts<ACT>(c[v], (float)x.e[v], (float)dy.e[v], h, dz);
                b[v] += dz;
                g[v] += dz * h;
            }
        };
        int64_t left = (t.rows - t.r + t.rpar - 1) / t.rpar;
        for (; left >= R; left -= R) {
            Pack<T, V> x[R], dy[R];
#pragma unroll
            for (int i = 0; i < R; ++i) { x[i] = load_pack<T, V>(p + i * xs); dy[i] = load_pack<T, V>(q + i * ys); }
#pragma unroll
            for (int i = 0; i < R; ++i) add(x[i], dy[i]);
            p += R * xs;
            q += R * ys;
        }
        for (; left > 0; --left, p += xs, q += ys) add(load_pack<T, V>(p), load_pack<T, V>(q));
    }
    float2 *chan = a.chan + ((size_t)t.n * a.chunks + t.s) * a.C + t.c0;
    float2 *part = a.part + (((size_t)t.n * a.tiles + t.t) * a.chunks + t.s) * (a.ct / a.D);
    const float *gamma = a.gamma ? a.gamma + t.c0 : nullptr;
    for (int k = 0; k < 2; ++k) {
        int nch, parts;
        const float *sums = column_sums<V>(t, k ? g : b, lds, &nch, &parts);
        for (int j = threadIdx.x; j < nch; j += blockDim.x) {
            float s = 0.f;
            for (int q = 0; q < parts; ++q) s += sums[q * nch + j];
            (k ? chan[j].y : chan[j].x) = s;
        }
        join_groups(sums, nch, parts, t.groups, a.D, gsum, [&](int ch) { return gamma ? gamma[ch] : 1.f; });
        __syncthreads();
        for (int j = threadIdx.x; j < t.groups; j += blockDim.x) (k ? part[j].y : part[j].x) = gsum[j];
    }
}

// dgamma, dbeta of 16 channels from the chunks' sums, added in a fixed order.
__device__ __forceinline__ void channel_grads(const NormArgs &a, int block, float *lds)
{
    const int ch = block * 16 + threadIdx.x % 16, r = threadIdx.x / 16, rows = blockDim.x / 16;
    float2 s = make_float2(0.f, 0.f);
    if (ch < a.C)
        for (int64_t i = r; i < a.N * a.chunks; i += rows) {
            const float2 v = a.chan[(size_t)i * a.C + ch];
            s.x += v.x;
            s.y += v.y;
        }
    lds[2 * threadIdx.x] = s.x;
    lds[2 * threadIdx.x + 1] = s.y;
    __syncthreads();
    if (r == 0 && ch < a.C) {
        for (int i = 1; i < rows; ++i) {
            s.x += lds[2 * (i * 16 + threadIdx.x)];
            s.y += lds[2 * (i * 16 + threadIdx.x) + 1];
        }
        if (a.dbeta) a.dbeta[ch] = s.x;
        if (a.dgamma) a.dgamma[ch] = s.y;
    }
}

// Second launch: dx, and in the workgroups behind those dgamma and dbeta.
template <typename T, int V, int ACT> __global__ __launch_bounds__(kMaxThreads) void norm_grad_apply_kernel(NormArgs a, uint32_t apply_blocks)
{
    constexpr int R = 2;
    extern __shared__ float lds[];
    if (blockIdx.x >= apply_blocks) {
        channel_grads(a, blockIdx.x - apply_blocks, lds);
        return;
    }
    const Tile t = find_tile<V>(a);
    const int gt = a.ct / a.D;
    const float2 *part = a.part + ((size_t)t.n * a.tiles + t.t) * a.chunks * gt;
    const int lane = threadIdx.x & 63, waves = blockDim.x / 64;
    const float inv = 1.f / ((float)a.P * (float)a.D);
    for (int g = threadIdx.x / 64; g < t.groups; g += waves) {
        float2 s = make_float2(0.f, 0.f);
        for (int i = lane; i < a.chunks; i += 64) {
            const float2 v = part[(size_t)i * gt + g];
            s.x += v.x;
            s.y += v.y;
        }
        for (int o = 32; o; o /= 2) { s.x += __shfl_xor(s.x, o); s.y += __shfl_xor(s.y, o); }
        if (lane == 0) { lds[2 * g] = s.x * inv; lds[2 * g + 1] = s.y * inv; }
    }
    __syncthreads();
    if (t.r >= t.rpar) return;
    Channel c[V];
    float sa[V], sb[V];
    load_channels<V>(a, t, c);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int g = (t.col * V + v) / a.D;
        sa[v] = lds[2 * g];
        sb[v] = lds[2 * g + 1];
    }
    const T *p = x_at<T, V>(a, t);
    const int64_t off = t.n * a.yn + (t.row0 + t.r) * a.yp + t.c0 + t.col * V;
    const T *q = (const T *)a.dy + off;
    T *w = (T *)a.dx + (p - (const T *)a.x);
    const int64_t xs = t.rpar * a.xp, ys = t.rpar * a.yp;
    auto one = [&](const Pack<T, V> &x, const Pack<T, V> &dy) {
        Pack<T, V> d;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float h, dz;
            grad_parts<ACT>(c[v], (float)x.e[v], (float)dy.e[v], h, dz);
            d.e[v] = (T)grad_input(c[v], h, dz, sa[v], sb[v]);
        }
        return d;
    };
    int64_t left = (t.rows - t.r + t.rpar - 1) / t.rpar;
    for (; left >= R; left -= R) {
        Pack<T, V> x[R], dy[R];
#pragma unroll
        for (int i = 0; i < R; ++i) { x[i] = load_pack<T, V>(p + i * xs); dy[i] = load_pack<T, V>(q + i * ys); }
#pragma unroll
        for (int i = 0; i < R; ++i) store_pack<T, V>(w + i * xs, one(x[i], dy[i]));
        p += R * xs;
        q += R * ys;
        w += R * xs;
    }
    for (; left > 0; --left, p += xs, q += ys, w += xs) store_pack<T, V>(w, one(load_pack<T, V>(p), load_pack<T, V>(q)));
}

// Zeros for dgamma and dbeta of no images.
__global__ void norm_zero_kernel(float *dgamma, float *dbeta, int C)
{
    const int c = blockIdx.x * blockDim.x + threadIdx.x;
    if (c < C && dgamma) dgamma[c] = 0.f;
    if (c < C && dbeta) dbeta[c] = 0.f;
}

NormArgs norm_args(const NormCall &c, const NormPlan &p, void *ws)
{
    NormArgs a{};
    a.x = c.x; a.dy = c.dy; a.y = c.y; a.dx = c.dx;
    a.gamma = c.gamma; a.beta = c.beta;
    a.mean = c.mean; a.rstd = c.rstd; a.dgamma = c.dgamma; a.dbeta = c.dbeta;
    a.N = c.d.N; a.P = c.d.P; a.rows = p.rows;
    a.xp = c.d.x_pixel; a.xn = c.d.x_image; a.yp = c.d.y_pixel; a.yn = c.d.y_image;
    a.C = c.d.C; a.G = c.d.groups; a.D = c.d.C / c.d.groups; a.ct = p.ct; a.tiles = p.tiles; a.chunks = p.chunks;
    a.eps = c.d.eps;
    a.part = (float2 *)ws;
    a.chan = a.part + (size_t)c.d.N * p.tiles * p.chunks * (p.ct / a.D);
    return a;
}

template <typename F> hipError_t with_width(int type, int V, F &&f)
{
    return with_type(type, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        if constexpr (sizeof(T) == 2) {
            if (V == 8) return f(null, std::integral_constant<int, 8>());
        }
        return V == 4 ? f(null, std::integral_constant<int, 4>()) : V == 2 ? f(null, std::integral_constant<int, 2>()) : f(null, std::integral_constant<int, 1>());
    });
}

template <typename F> hipError_t with_act(int act, F &&f)
{
    return act == QRM_ACT_SILU ? f(std::integral_constant<int, QRM_ACT_SILU>())
           : act == QRM_ACT_RELU ? f(std::integral_constant<int, QRM_ACT_RELU>()) : f(std::integral_constant<int, QRM_ACT_NONE>());
}

} // namespace

bool plan_norm(const qrm_group_norm_desc &d, int align_bytes, bool backward, int num_cu, NormPlan *out)
{
    const int size = type_bytes(d.type), D = d.C / d.groups;
    NormPlan p{};
    // the widest piece that the addresses, the strides and the number of channels allow
    p.V = std::min(16, align_bytes) / size;
    while (d.C % p.V || d.x_pixel % p.V || d.y_pixel % p.V || d.x_image % p.V || d.y_image % p.V) p.V /= 2;
    int64_t unit = std::lcm<int64_t>(D, p.V);
    if (unit / p.V > 256) { // (pieces that straddle groups: the shared memory holds 256 of them)
        p.V = std::gcd(D, p.V);
        unit = D;
    }
    if (unit / p.V > kMaxThreads) return false;
    p.uniform = D % p.V == 0;
    const int64_t lines = std::max<int64_t>(1, (128 + unit * size - 1) / (unit * size)); // units to a 128-byte line
    p.ct = (int)std::min<int64_t>(d.C, lines * unit);
    p.tiles = (d.C + p.ct - 1) / p.ct;
    const int cols = p.ct / p.V;
    p.threads = std::max(256, (cols + 63) / 64 * 64);
    const int rpar = p.threads / cols;
    // four workgroups to a compute unit where each has at least eight pixels a thread
    const int64_t want = std::max<int64_t>(1, 4LL * num_cu / std::max<int64_t>(1, d.N * p.tiles));
    const int64_t most = std::max<int64_t>(1, d.P / (8LL * rpar));
    const int64_t chunks = std::min(want, most);
    p.rows = (d.P + chunks - 1) / chunks;
    p.chunks = (int)((d.P + p.rows - 1) / p.rows);
    p.bytes = (size_t)d.N * p.tiles * p.chunks * (p.ct / D) * sizeof(float2);
    if (backward) p.bytes += (size_t)d.N * p.chunks * d.C * sizeof(float2);
    *out = p;
    return true;
}

hipError_t launch_norm_forward(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s)
{
    const NormArgs a = norm_args(c, p, ws);
    const dim3 grid((uint32_t)(c.d.N * p.tiles * p.chunks)), block(p.threads);
    const int gt = p.ct / a.D;
    return with_width(c.d.type, p.V, [&](auto *null, auto width) {
        using T = std::remove_pointer_t<decltype(null)>;
        constexpr int V = decltype(width)::value;
        if (p.uniform)
            hipLaunchKernelGGL((norm_stats_kernel<T, V, true>), grid, block, (sum_floats(p.threads, 1) + gt) * sizeof(float), s, a);
        else
            hipLaunchKernelGGL((norm_stats_kernel<T, V, false>), grid, block, (sum_floats(p.threads, V) + gt) * sizeof(float), s, a);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        return with_act(c.d.act, [&](auto act) {
            hipLaunchKernelGGL((norm_apply_kernel<T, V, decltype(act)::value>), grid, block, 2 * gt * sizeof(float), s, a);
            return hipGetLastError();
        });
    });
}

hipError_t launch_norm_backward(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s)
{
    if (c.d.N == 0) {
        hipLaunchKernelGGL(norm_zero_kernel, dim3((c.d.C + 255) / 256), dim3(256), 0, s, c.dgamma, c.dbeta, c.d.C);
        return hipGetLastError();
    }
    const NormArgs a = norm_args(c, p, ws);
    const uint32_t blocks = (uint32_t)(c.d.N * p.tiles * p.chunks);
    const int gt = p.ct / a.D;
    return with_width(c.d.type, p.V, [&](auto *null, auto width) {
        using T = std::remove_pointer_t<decltype(null)>;
        constexpr int V = decltype(width)::value;
        return with_act(c.d.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            hipLaunchKernelGGL((norm_grad_sums_kernel<T, V, ACT>), dim3(blocks), dim3(p.threads), (sum_floats(p.threads, V) + gt) * sizeof(float), s, a);
            hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            const uint32_t apply = c.dx ? blocks : 0, extra = c.dgamma || c.dbeta ? (c.d.C + 15) / 16 : 0;
            hipLaunchKernelGGL((norm_grad_apply_kernel<T, V, ACT>), dim3(apply + extra), dim3(p.threads), 2 * std::max(gt, p.threads) * sizeof(float), s, a, apply);
            return hipGetLastError();
        });
    });
}

} // namespace qrm
