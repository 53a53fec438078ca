// Attention: how a call is cut into launches, and the kernels around the matrix products that read and write rows one by one (those: attention.h).
#include "qrm_train.h"

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>

namespace qrm {

hipError_t launch_attention_f32(int kind, const AttnArgs &a, hipStream_t s);
hipError_t launch_attention_bf16(int kind, const AttnArgs &a, hipStream_t s);
hipError_t launch_attention_f16(int kind, const AttnArgs &a, hipStream_t s);

namespace {

constexpr int kThreads = 256;
constexpr float kLn2 = 0.693147180559945309f;

uint32_t blocks_of(int64_t items) { return (uint32_t)((items + kThreads - 1) / kThreads); }

// Sixteen lanes a row: minus the sum of dy o, and minus the log-sum over the scale (a row that sees nothing: -inf, so that its probabilities are zeros).
// Rows behind an image's queries are not read.
constexpr int kRowLanes = 16;
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void attention_rows_kernel(const T *o, const T *dy, int64_t row, int64_t head, int64_t image, const float *lse, const int32_t *q_len,
                                                                  int64_t all, int Lq, int heads, int D, float scale, float *row_lse, float *row_delta)
{
    const int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / kRowLanes;
    const int lane = threadIdx.x % kRowLanes;
    if (i >= all) return;
    const int64_t n = i / ((int64_t)heads * Lq);
    const int rest = (int)(i - n * heads * Lq), h = rest / Lq, pos = rest % Lq;
    const bool there = !q_len || pos < q_len[n];
    float sum = 0.f;
    if (there) {
        const int64_t at = n * image + h * head + pos * row;
        for (int d = lane * V; d < D; d += kRowLanes * V) {
            const Pack<T, V> x = load_pack<T, V>(o + at + d), y = load_pack<T, V>(dy + at + d);
#pragma unroll
            for (int e = 0; e < V; ++e) sum = __builtin_fmaf((float)x.e[e], (float)y.e[e], sum);
        }
    }
    for (int apart = kRowLanes / 2; apart; apart /= 2) sum += __shfl_xor(sum, apart);
    if (lane == 0) {
        const float l = there ? lse[i] : -INFINITY;
        row_lse[i] = l == -INFINITY ? -INFINITY : -l / scale;
        row_delta[i] = l == -INFINITY ? 0.f : -sum;
    }
}

// Joins the splits of a row: a thread has four elements of some of them; `lanes` threads, a power of two, have the same elements of others.  A row that was
// written at once is left alone.
struct JoinCut {
    int quads, lanes, rows; // threads to a split's row (a power of two), of the same elements, rows of a workgroup
    uint32_t blocks(int64_t all) const { return (uint32_t)((all + rows - 1) / rows); }
};
JoinCut join_cut(int D, int splits)
{
    JoinCut c{1, 1, 0};
    while (c.quads * 4 < D) c.quads *= 2;
    while (c.lanes < splits && c.lanes * c.quads < kThreads) c.lanes *= 2;
    c.rows = kThreads / (c.quads * c.lanes);
    return c;
}

// Adds f32 sums of `lanes` threads that are `quads` threads apart; the first has them.
template <int COUNT> __device__ __forceinline__ void add_lanes(float (&v)[COUNT], int quads, int lanes, float (*shared)[COUNT + 1])
{
    for (int apart = lanes / 2; apart; apart /= 2) {
        if (apart * quads < 64 && quads * apart * 2 <= 64) {
#pragma unroll
            for (int e = 0; e < COUNT; ++e) v[e] += __shfl_down(v[e], apart * quads);
        } else {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < COUNT; ++e) shared[threadIdx.x][e] = v[e];
            __syncthreads();
            const int from = threadIdx.x + apart * quads;
            if (from < kThreads)
#pragma unroll
                for (int e = 0; e < COUNT; ++e) v[e] += shared[from][e];
        }
    }
}

// The forward's: results about a power of two, and their sum.
template <typename T> __global__ __launch_bounds__(kThreads) void attention_join_kernel(AttnArgs a, JoinCut cut, int64_t all)
{
    __shared__ float shared[kThreads][6];
    const int quad = threadIdx.x % cut.quads, lane = threadIdx.x / cut.quads % cut.lanes, d = quad * 4;
    const int64_t i = (int64_t)blockIdx.x * cut.rows + threadIdx.x / (cut.quads * cut.lanes);
    const int64_t n = min(i, all - 1) / ((int64_t)a.heads * a.Lq);
    const int rest = (int)(min(i, all - 1) - n * a.heads * a.Lq), h = rest / a.Lq, pos = rest % a.Lq;
    const int part = (pos * a.group + h % a.group) / a.columns;
    const int splits = attn_split(attn_key_tiles(a, attn_length(a.q_len, n, a.Lq), attn_length(a.k_len, n, a.Lk), part), a.per, 0).count;
    const bool mine = i < all && splits > 1;
    const float2 *const sums = (const float2 *)a.part_sums;
    float top = -INFINITY;
    if (mine)
        for (int k = 0; k < splits; ++k) top = fmaxf(top, sums[k * all + i].x);
    float o[5] = {}; // .. and the sum
    if (mine && d < a.D)
#pragma unroll 4
        for (int k = lane; k < splits; k += cut.lanes) {
            const float2 s = sums[k * all + i];
            const Pack<float, 4> p = load_pack<float, 4>(a.part + (k * all + i) * a.D + d);
            const float by = s.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s.x - top);
            o[4] += s.y * by;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += by == 0.f ? 0.f : p.e[e] * by;
        }
    add_lanes<5>(o, cut.quads, cut.lanes, shared);
    if (!mine || lane || d >= a.D) return;
    const bool some = top != -INFINITY;
    const float inv = some ? 1.f / o[4] : 0.f;
    Pack<T, 4> out;
#pragma unroll
    for (int e = 0; e < 4; ++e) out.e[e] = (T)(o[e] * inv);
    store_pack<T, 4>((T *)a.o + n * a.o_image + h * a.o_head + pos * a.o_row + d, out);
    if (d == 0 && a.lse) a.lse[i] = some ? (top + __builtin_amdgcn_logf(o[4])) * kLn2 : -INFINITY;
}

// Gradients': dq's rows, then those of dk, then those of dv.
struct AddJob {
    const float *part;
    void *out;
    int64_t row, head, image, all;
    uint32_t first; // workgroup
    JoinCut cut;
};
template <typename T> __global__ __launch_bounds__(kThreads) void attention_add_kernel(AttnArgs by_q, AttnArgs by_k, AddJob q, AddJob k, AddJob v)
{
    __shared__ float shared[kThreads][5];
    const bool is_q = blockIdx.x < k.first;
    const AttnArgs &a = is_q ? by_q : by_k;
    const AddJob j = is_q ? q : blockIdx.x < v.first ? k : v;
    const int quad = threadIdx.x % j.cut.quads, lane = threadIdx.x / j.cut.quads % j.cut.lanes, d = quad * 4;
    const int64_t i = (int64_t)(blockIdx.x - j.first) * j.cut.rows + threadIdx.x / (j.cut.quads * j.cut.lanes), near = min(i, j.all - 1);
    const int L = is_q ? a.Lq : a.Lk, heads = is_q ? a.heads : a.kv_heads;
    const int64_t n = near / ((int64_t)heads * L);
    const int rest = (int)(near - n * heads * L), h = rest / L, pos = rest % L;
    const int q_len = attn_length(a.q_len, n, a.Lq), k_len = attn_length(a.k_len, n, a.Lk);
    int skip;
    const int tiles = is_q ? attn_key_tiles(a, q_len, k_len, (pos * a.group + h % a.group) / a.columns) : attn_query_tiles(a, q_len, k_len, pos / a.columns, &skip) * a.group;
    const int splits = attn_split(tiles, a.per, 0).count;
    const bool mine = i < j.all && splits > 1;
    float sum[4] = {};
    if (mine && d < a.D)
#pragma unroll 4
        for (int s = lane; s < splits; s += j.cut.lanes) {
            const Pack<float, 4> p = load_pack<float, 4>(j.part + (s * j.all + i) * a.D + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += p.e[e];
        }
    add_lanes<4>(sum, j.cut.quads, j.cut.lanes, shared);
    if (!mine || lane || d >= a.D) return;
    Pack<T, 4> out;
#pragma unroll
    for (int e = 0; e < 4; ++e) out.e[e] = (T)sum[e];
    store_pack<T, 4>((T *)j.out + n * j.image + h * j.head + pos * j.row + d, out);
}

// Rows [N,L,heads,D] from one place to another, element by element on the side that is not aligned: into rows of `wide` elements, zeros behind the D, or
// out of such.
template <typename T, bool OUT>
__global__ __launch_bounds__(kThreads) void attention_copy_kernel(AttnRows rows, T *there, T *here, int64_t all, int64_t L, int heads, int D, int wide)
{
    constexpr int E = 16 / (int)sizeof(T);
    const int pieces = wide / E;
    const int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x, i = t / pieces;
    if (i >= all) return;
    const int d = (int)(t - i * pieces) * E;
    const int64_t nh = i / L;
    T *const far = there + nh / heads * rows.image + nh % heads * rows.head + (i - nh * L) * rows.row;
    Pack<T, E> v = {};
    if (OUT) v = load_pack<T, E>(here + i * wide + d);
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (d + e < D) {
            if (OUT) far[d + e] = v.e[e];
            else v.e[e] = far[d + e];
        }
    if (!OUT) store_pack<T, E>(here + i * wide + d, v);
}

} // namespace

hipError_t launch_attention(int type, int kind, const AttnArgs &a, hipStream_t s)
{
    return type == QRM_F32 ? launch_attention_f32(kind, a, s) : type == QRM_BF16 ? launch_attention_bf16(kind, a, s) : launch_attention_f16(kind, a, s);
}

hipError_t launch_attention_rows(const qrm_attention_desc &d, const void *o, const void *dy, const float *lse, const int32_t *q_len, float *row_lse, float *row_delta, hipStream_t s)
{
    const int64_t all = d.N * d.heads * d.Lq;
    const int size = type_bytes(d.type), v = 16 / size;
    const bool wide = ((uintptr_t)o | (uintptr_t)dy) % 16 == 0 && d.D % v == 0 && d.o_row % v == 0 && d.o_head % v == 0 && d.o_image % v == 0;
    const dim3 grid(blocks_of(all * kRowLanes));
    return with_type(d.type, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        auto run = [&](auto width) {
            hipLaunchKernelGGL((attention_rows_kernel<T, decltype(width)::value>), grid, dim3(kThreads), 0, s, (const T *)o, (const T *)dy, d.o_row, d.o_head, d.o_image, lse, q_len,
                               all, (int)d.Lq, d.heads, d.D, d.scale, row_lse, row_delta);
        };
        wide ? run(std::integral_constant<int, 16 / sizeof(T)>()) : run(std::integral_constant<int, 1>());
        return hipGetLastError();
    });
}

hipError_t launch_attention_join(int type, const AttnArgs &a, hipStream_t s)
{
    const int64_t all = (int64_t)a.N * a.heads * a.Lq;
    const JoinCut cut = join_cut(a.D, a.splits);
    return with_type(type, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        hipLaunchKernelGGL((attention_join_kernel<T>), dim3(cut.blocks(all)), dim3(kThreads), 0, s, a, cut, all);
        return hipGetLastError();
    });
}

hipError_t launch_attention_add(int type, const AttnArgs &by_q, const AttnArgs &by_k, hipStream_t s)
{
    uint32_t blocks = 0;
    auto job = [&](const AttnArgs &a, const float *part, void *out, int64_t row, int64_t head, int64_t image, int64_t all) {
        AddJob j{part, out, row, head, image, all, blocks, join_cut(a.D, a.splits)};
        if (out && a.splits > 1) blocks += j.cut.blocks(all);
        return j;
    };
    const AddJob q = job(by_q, by_q.part, by_q.dq, by_q.q_row, by_q.q_head, by_q.q_image, (int64_t)by_q.N * by_q.heads * by_q.Lq);
    const int64_t keys = (int64_t)by_k.N * by_k.kv_heads * by_k.Lk;
    const AddJob k = job(by_k, by_k.part_k, by_k.dk, by_k.k_row, by_k.k_head, by_k.k_image, keys), v = job(by_k, by_k.part_v, by_k.dv, by_k.v_row, by_k.v_head, by_k.v_image, keys);
    if (!blocks) return hipSuccess;
    return with_type(type, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        hipLaunchKernelGGL((attention_add_kernel<T>), dim3(blocks), dim3(kThreads), 0, s, by_q, by_k, q, k, v);
        return hipGetLastError();
    });
}

hipError_t launch_attention_copy(int type, bool out, const AttnRows &r, void *there, void *here, int64_t N, int64_t L, int heads, int D, int wide, hipStream_t s)
{
    const int64_t all = N * heads * L;
    const int E = 16 / type_bytes(type);
    return with_type(type, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        const dim3 grid(blocks_of(all * (wide / E)));
        if (out) hipLaunchKernelGGL((attention_copy_kernel<T, true>), grid, dim3(kThreads), 0, s, r, (T *)there, (T *)here, all, L, heads, D, wide);
        else hipLaunchKernelGGL((attention_copy_kernel<T, false>), grid, dim3(kThreads), 0, s, r, (T *)there, (T *)here, all, L, heads, D, wide);
        return hipGetLastError();
    });
}

// Splits of the other side are as many as let the busiest compute unit be done first, by a model of times in us: tiles at the rate that the kernels reach
// (0.4 of the matrix products' peak), a workgroup alone on its compute unit at 0.65 of the time that it takes beside others, 3 us for a workgroup's beginning and
// end, and the join, a launch that reads what the splits write.
AttnCut plan_attention(const qrm_attention_desc &d, int width, int kind, int num_cu)
{
    const int size = type_bytes(d.type), w = attn_width(width);
    const int64_t group = d.heads / d.kv_heads, columns = kind == ATTN_DKV ? d.Lk : d.Lq * group, others = kind == ATTN_DKV ? d.Lq : d.Lk;
    AttnCut c{};
    c.kind = kind;
    if (kind == ATTN_FORWARD && columns <= attn_shape(size, w, ATTN_FEW).rows()) c.kind = ATTN_FEW;
    const AttnShape h = c.shape = attn_shape(size, w, c.kind);
    c.parts = (int)((columns + h.rows() - 1) / h.rows());
    const int64_t tiles = std::max<int64_t>(1, (others + h.tile - 1) / h.tile * (kind == ATTN_DKV ? group : 1)), blocks = std::max<int64_t>(1, d.N * d.kv_heads * c.parts);
    // the share of the tiles that a part sees on average where causal: of Lq x Lk, all but a triangle
    const double lq = (double)d.Lq, lk = (double)d.Lk, seen = std::min(lq, lk), share = !d.causal || lq * lk == 0.0 ? 1.0 : seen * (lk - 0.5 * seen) / (lq * lk);
    const double products = kind == ATTN_FORWARD ? 2.0 : kind == ATTN_DQ ? 3.0 : 4.0, rate = (size == 2 ? 1e15 : 6e13) / num_cu * 1e-6; // operations in a us of a compute unit
    const double tile_us = products * 2.0 * h.rows() * h.tile * w / rate;
    const double part_us = (kind == ATTN_DKV ? 2.0 : 1.0) * d.N * d.kv_heads * (double)columns * width * 8.0 / 4e6; // written and read again, a split
    double best = 0.0;
    for (int64_t n = 1; n <= std::min<int64_t>(tiles, 64); ++n) {
        const int64_t per = (tiles + n - 1) / n;
        if ((tiles + per - 1) / per != n) continue;
        const double all = std::max(1.0, n * share + (n > 1 && share < 1.0 ? 0.5 : 0.0)) * blocks, on_one = std::ceil(all / num_cu);
        const double rounds = std::floor(on_one / h.occupancy) + 0.65 * (std::fmod(on_one, h.occupancy) > 0.0 ? 1.0 : 0.0);
        const double us = rounds * (std::min(per * 1.0, tiles * share) * tile_us * h.occupancy + 3.0) + (n > 1 ? 5.0 + part_us * n * share : 0.0);
        if (n == 1 || us < best) best = us, c.splits = (int)n, c.per = (int)per;
    }
    const char *env = getenv(kind == ATTN_DKV ? "SPL_K" : kind == ATTN_DQ ? "SPL_Q" : "SPL_F");
    if (env) {
        const int64_t n = std::min<int64_t>(atoi(env), tiles);
        c.per = (int)((tiles + n - 1) / n);
        c.splits = (int)((tiles + c.per - 1) / c.per);
    }
    if (getenv("SPL_SAY")) printf("kind %d blocks %ld tiles %ld splits %d per %d tile_us %.2f\n", c.kind, (long)blocks, (long)tiles, c.splits, c.per, tile_us);
    return c;
}

} // namespace qrm
