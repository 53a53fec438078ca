// Attention: how a call is cut into launches, and the kernels around the matrix products that read and write rows one by one (those: attention.h).
#include "qrm_train.h"

#include <algorithm>
#include <cmath>

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

// Joins the splits of a forward pass: a thread has four elements of a row.
template <typename T> __global__ __launch_bounds__(kThreads) void attention_join_kernel(AttnArgs a, int64_t all)
{
    const int quads = a.D / 4;
    const int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x, i = t / quads;
    if (i >= all) return;
    const int d = (int)(t - i * quads) * 4;
    const float2 *const sums = (const float2 *)a.part_sums;
    float top = -INFINITY;
    for (int k = 0; k < a.splits; ++k) top = fmaxf(top, sums[k * all + i].x);
    float sum = 0.f, o[4] = {};
    for (int k = 0; k < a.splits; ++k) {
        const float2 s = sums[k * all + i];
        const Pack<float, 4> p = load_pack<float, 4>(a.part + (k * all + i) * a.D + d);
        if (s.x == -INFINITY) continue;
        const float by = __builtin_amdgcn_exp2f(s.x - top);
        sum += s.y * by;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(p.e[e], by, o[e]);
    }
    const bool some = top != -INFINITY;
    const float inv = some ? 1.f / sum : 0.f;
    const int64_t n = i / ((int64_t)a.heads * a.Lq);
    const int rest = (int)(i - n * a.heads * a.Lq), h = rest / a.Lq, pos = rest % a.Lq;
    Pack<T, 4> out;
#pragma unroll
    for (int e = 0; e < 4; ++e) out.e[e] = (T)(o[e] * inv);
    store_pack<T, 4>((T *)a.o + n * a.o_image + h * a.o_head + pos * a.o_row + d, out);
    if (d == 0 && a.lse) a.lse[i] = some ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
}

// Sums of gradient parts [splits][N,heads,L,D].
template <typename T>
__global__ __launch_bounds__(kThreads) void attention_add_kernel(const float *part, int splits, T *out, int64_t all, int64_t L, int heads, int D, int64_t row, int64_t head, int64_t image)
{
    const int quads = D / 4;
    const int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x, i = t / quads;
    if (i >= all) return;
    const int d = (int)(t - i * quads) * 4;
    float sum[4] = {};
    for (int k = 0; k < splits; ++k) {
        const Pack<float, 4> p = load_pack<float, 4>(part + (k * all + i) * D + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += p.e[e];
    }
    const int64_t nh = i / L;
    Pack<T, 4> v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v.e[e] = (T)sum[e];
    store_pack<T, 4>(out + nh / heads * image + nh % heads * head + (i - nh * L) * row + d, v);
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
    return with_type(type, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        hipLaunchKernelGGL((attention_join_kernel<T>), dim3(blocks_of(all * (a.D / 4))), dim3(kThreads), 0, s, a, all);
        return hipGetLastError();
    });
}

hipError_t launch_attention_add(int type, const float *part, int splits, void *out, const AttnRows &r, int64_t N, int64_t L, int heads, int D, hipStream_t s)
{
    const int64_t all = N * heads * L;
    return with_type(type, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        hipLaunchKernelGGL((attention_add_kernel<T>), dim3(blocks_of(all * (D / 4))), dim3(kThreads), 0, s, part, splits, (T *)out, all, L, heads, D, r.row, r.head, r.image);
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

AttnCut plan_attention(const qrm_attention_desc &d, int width, int kind, int num_cu)
{
    const int size = type_bytes(d.type), w = attn_width(width);
    const int64_t group = d.heads / d.kv_heads, columns = kind == ATTN_DKV ? d.Lk : d.Lq * group, others = kind == ATTN_DKV ? d.Lq : d.Lk;
    AttnCut c{};
    c.kind = kind;
    if (kind == ATTN_FORWARD && columns <= attn_shape(size, w, ATTN_FEW).rows()) c.kind = ATTN_FEW;
    const AttnShape h = attn_shape(size, w, c.kind);
    c.parts = (int)((columns + h.rows() - 1) / h.rows());
    const int64_t tiles = (others + h.tile - 1) / h.tile * (kind == ATTN_DKV ? group : 1), blocks = d.N * d.kv_heads * c.parts;
    const int64_t want = (int64_t)num_cu * (c.kind == ATTN_FEW ? 4 : h.occupancy);
    c.splits = (int)std::max<int64_t>(1, std::min<int64_t>({blocks ? want / blocks : 1, tiles / 4, 64}));
    return c;
}

} // namespace qrm
