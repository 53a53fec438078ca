// Attention: how a call is cut into launches, and the kernels around the matrix products that read and write rows one by one (those: attention.h).
#include "qrm_train.h"

#include <algorithm>
#include <cmath>

namespace qrm {

hipError_t launch_attention_f32(int kind, const AttnArgs &a, hipStream_t s);
hipError_t launch_attention_bf16(int kind, const AttnArgs &a, hipStream_t s);
hipError_t launch_attention_f16(int kind, const AttnArgs &a, hipStream_t s);
hipError_t launch_attention_backward_f32(const AttnArgs &by_q, const AttnArgs &by_k, hipStream_t s);
hipError_t launch_attention_backward_bf16(const AttnArgs &by_q, const AttnArgs &by_k, hipStream_t s);
hipError_t launch_attention_backward_f16(const AttnArgs &by_q, const AttnArgs &by_k, hipStream_t s);

namespace {

constexpr int kThreads = 256;
constexpr float kLog2E = 1.44269504088896341f;

uint32_t blocks_of(int64_t items) { return (uint32_t)((items + kThreads - 1) / kThreads); }

// Sixteen lanes a row: minus the sum of dy o, and minus the log-sum over the scale (a row that sees nothing: -inf, so that its probabilities are zeros).
// Rows behind an image's queries are not read.  Bound by memory: 131072 rows of 128 elements of bf16, 67 MB, in 16 us, 4.2 TB/s.
constexpr int kRowLanes = 16;
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void attention_rows_kernel(const T *o, const T *dy, int64_t row, int64_t head, int64_t image, const float *lse, const int32_t *q_len,
                                                                  int all, Quotient by_heads, Quotient by_rows, int D, float scale, float *row_lse, float *row_delta)
{
    const int i = (int)((blockIdx.x * kThreads + threadIdx.x) / kRowLanes), lane = threadIdx.x % kRowLanes;
    if (i >= all) return;
    const int head_of = by_rows.of(i), pos = i - head_of * (int)by_rows.by, n = by_heads.of(head_of), h = head_of - n * (int)by_heads.by;
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

// Joins the splits of a launch: a thread has two times four results of a row, where the lanes of the splits' workgroups had them (store_part).  What was written at
// once is left alone.  Bound by memory (most of it in the last cache), if enough is on its way: kAhead splits are read before the first of them is added, and what
// does not depend on the lane is computed once a wavefront (one head of 512, 4 x 4096
// rows in 2 splits, 67 MB: 16 us, 5.2 TB/s; one block a thread, split after split and with divisions 23).
struct JoinTo {
    const float *part;
    void *out;
    int64_t row, head, image;
    uint32_t first; // workgroup
};
struct JoinJob {
    JoinTo to;
    AttnShape shape;
    int width, pairs;             // pairs of blocks of a part: a block is what 64 lanes hold in four registers
    Quotient by_pairs, by_blocks; // by_blocks: of a wavefront
};
constexpr int kAhead = 4;
// KEYS: rows are those of keys.  SUMS: forward, (raw score that a row's results are about, their sum).
template <typename T, bool KEYS, bool SUMS> __device__ __forceinline__ void join_part(const AttnArgs &a, const JoinJob &j, const JoinTo &to)
{
    const AttnShape &h = j.shape;
    const int unit = __builtin_amdgcn_readfirstlane((blockIdx.x - to.first) * (kThreads / 64) + threadIdx.x / 64), which = j.by_pairs.of(unit), lane = threadIdx.x % 64;
    const int group = a.by_parts.of(which), part = which - group * a.parts, n = a.by_kv_heads.of(group), kv = group - n * a.kv_heads;
    if (n >= a.N) return;
    const int q_len = attn_length(a.q_len, n, a.Lq), k_len = attn_length(a.k_len, n, a.Lk);
    int skip;
    const int tiles = KEYS ? attn_query_tiles(a, q_len, k_len, part, &skip) * a.group : attn_key_tiles(a, q_len, k_len, part);
    const int splits = attn_split(a, tiles, 0).count;
    if (splits == 1) return;
    // the lane's column and elements: as in store_part and Mma::row_of
    const int pair = unit - which * j.pairs, ng = 64 / h.m, quads = h.m * h.m / 256, each = j.width / h.share, blocks = each / h.m * quads;
    const int wave = j.by_blocks.of(pair * 2), block = pair * 2 - wave * blocks, column = wave / h.share * h.m + lane % h.m;
    const int r = part * a.columns + column, pos = KEYS ? r : attn_position(a, r), head = KEYS ? kv : kv * a.group + (r - pos * a.group);
    if (pos >= (KEYS ? a.Lk : a.Lq)) return;
    const int64_t apart = (int64_t)a.N * a.kv_heads * a.parts; // slots from one split to the next
    const f32x4 *const from = (const f32x4 *)to.part + ((int64_t)which * j.pairs + pair) * 128 + lane;
    f32x4 o[2] = {};
    float by_sum = 1.f;
    if constexpr (SUMS) {
        const float2 *const sums = (const float2 *)a.part_sums + which * (int64_t)a.columns + column;
        const float c = a.scale * kLog2E, lift = attn_lift(std::is_same<T, f16_t>::value);
        float top = -INFINITY, sum = 0.f; // (one pass: a split's sums and its results are on their way together)
        for (int k0 = 0; k0 < splits; k0 += kAhead) {
            float2 s[kAhead];
            f32x4 p[kAhead][2];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (k0 + i >= splits) break;
                const int64_t k = k0 + i;
                s[i] = sums[k * apart * a.columns];
                p[i][0] = from[k * apart * j.pairs * 128];
                p[i][1] = from[k * apart * j.pairs * 128 + 64];
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (k0 + i >= splits) break;
                const float now = fmaxf(top, s[i].x), less = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((top - now) * c), by = s[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((s[i].x - now) * c);
                top = now;
                sum = sum * less + s[i].y * by;
                // (a split of which the row sees nothing adds nothing; one of no weight beside the others adds zeros, and what is not finite stays so)
                const bool none = s[i].x == -INFINITY;
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e / 4][e % 4] = o[e / 4][e % 4] * less + (none ? 0.f : p[i][e / 4][e % 4] * by);
            }
        }
        const bool sees = pos < q_len && (a.causal ? min(k_len, pos + k_len - q_len + 1) : k_len) > 0;
        const float lse = sees ? attn_log_sum(top, a.scale, sum, lift) : -INFINITY;
        by_sum = sees ? lse == lse ? 1.f / sum : lse : 0.f;
        if (block == 0 && lane < h.m && wave % h.share == 0 && a.lse) a.lse[((int64_t)n * a.heads + head) * a.Lq + pos] = lse;
    } else if (!KEYS || r < k_len) {
        for (int k0 = 0; k0 < splits; k0 += kAhead) {
            f32x4 p[kAhead][2];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (k0 + i >= splits) break;
                const int64_t k = k0 + i;
                p[i][0] = from[k * apart * j.pairs * 128];
                p[i][1] = from[k * apart * j.pairs * 128 + 64];
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (k0 + i >= splits) break;
                o[0] += p[i][0], o[1] += p[i][1];
            }
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int d = wave % h.share * each + (block + u) / quads * h.m + ((block + u) % quads * ng + lane / h.m) * 4;
        Pack<T, 4> out;
#pragma unroll
        for (int e = 0; e < 4; ++e) out.e[e] = (T)(o[u][e] * by_sum);
        if (d < a.D) store_pack<T, 4>((T *)to.out + n * to.image + head * to.head + pos * to.row + d, out);
    }
}
template <typename T> __global__ __launch_bounds__(kThreads) void attention_join_kernel(AttnArgs a, JoinJob j) { join_part<T, false, true>(a, j, j.to); }
// (dk and dv by one copy of the code, and arguments of less than 1 KB: a backward pass of 4 x 256 rows of 4 heads 18.1 -> 17.7 us)
template <typename T> __global__ __launch_bounds__(kThreads) void attention_add_kernel(AttnArgs by_q, AttnArgs by_k, JoinJob q, JoinJob k, JoinTo v)
{
    const bool values = blockIdx.x >= v.first;
    if (blockIdx.x < k.to.first) join_part<T, false, false>(by_q, q, q.to);
    else join_part<T, true, false>(by_k, k, JoinTo{values ? v.part : k.to.part, values ? v.out : k.to.out, values ? v.row : k.to.row, values ? v.head : k.to.head,
                                                   values ? v.image : k.to.image, values ? v.first : k.to.first});
}

// Rows [N,L,heads,D] from one place to another, element by element on the side that is not aligned: into rows of `wide` elements, zeros behind the D, or
// out of such.  Bound by launches and single-element accesses: bf16, 2 x 2048 rows of 16 heads of
// 128 all an element off, forward 88 -> 130 us, backward 234 -> 329; 4 x 1024 rows of 8 heads of 64, 17 -> 40 and 41 -> 78.
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

hipError_t launch_attention_backward(int type, const AttnArgs &by_q, const AttnArgs &by_k, hipStream_t s)
{
    return type == QRM_F32 ? launch_attention_backward_f32(by_q, by_k, s) : type == QRM_BF16 ? launch_attention_backward_bf16(by_q, by_k, s) : launch_attention_backward_f16(by_q, by_k, s);
}

hipError_t launch_attention_rows(const qrm_attention_desc &d, const void *o, const void *dy, const float *lse, const int32_t *q_len, float *row_lse, float *row_delta, hipStream_t s)
{
    const int64_t all = d.N * d.heads * d.Lq; // (below 2^28: sixteen threads each)
    const int size = type_bytes(d.type), v = 16 / size;
    const bool wide = ((uintptr_t)o | (uintptr_t)dy) % 16 == 0 && d.D % v == 0 && d.o_row % v == 0 && d.o_head % v == 0 && d.o_image % v == 0;
    const dim3 grid(blocks_of(all * kRowLanes));
    return with_type(d.type, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        auto run = [&](auto width) {
            hipLaunchKernelGGL((attention_rows_kernel<T, decltype(width)::value>), grid, dim3(kThreads), 0, s, (const T *)o, (const T *)dy, d.o_row, d.o_head, d.o_image, lse, q_len,
                               (int)all, Quotient((uint32_t)d.heads), Quotient((uint32_t)d.Lq), d.D, d.scale, row_lse, row_delta);
        };
        wide ? run(std::integral_constant<int, 16 / sizeof(T)>()) : run(std::integral_constant<int, 1>());
        return hipGetLastError();
    });
}

namespace {

// Adds a job's workgroups to those that there are.
JoinJob join_job(const AttnArgs &a, const AttnCut &cut, const float *part, void *out, int64_t row, int64_t head, int64_t image, uint32_t *blocks)
{
    JoinJob j{{part, out, row, head, image, *blocks}, cut.shape, cut.width, cut.shape.rows() * cut.width / 512, Quotient(), Quotient()};
    const int m = cut.shape.m;
    j.by_pairs = Quotient(j.pairs), j.by_blocks = Quotient(cut.width / cut.shape.share / m * (m * m / 256));
    if (out && a.splits > 1) *blocks += blocks_of((int64_t)j.pairs * a.N * a.kv_heads * a.parts * 64);
    return j;
}

} // namespace

hipError_t launch_attention_join(int type, const AttnArgs &a, const AttnCut &cut, hipStream_t s)
{
    uint32_t blocks = 0;
    const JoinJob j = join_job(a, cut, a.part, a.o, a.o_row, a.o_head, a.o_image, &blocks);
    if (!blocks) return hipSuccess;
    return with_type(type, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        hipLaunchKernelGGL((attention_join_kernel<T>), dim3(blocks), dim3(kThreads), 0, s, a, j);
        return hipGetLastError();
    });
}

hipError_t launch_attention_add(int type, const AttnArgs &by_q, const AttnCut &cut_q, const AttnArgs &by_k, const AttnCut &cut_k, hipStream_t s)
{
    uint32_t blocks = 0;
    const JoinJob q = join_job(by_q, cut_q, by_q.part, by_q.dq, by_q.q_row, by_q.q_head, by_q.q_image, &blocks);
    const JoinJob k = join_job(by_k, cut_k, by_k.part_k, by_k.dk, by_k.k_row, by_k.k_head, by_k.k_image, &blocks);
    const JoinJob v = join_job(by_k, cut_k, by_k.part_v, by_k.dv, by_k.v_row, by_k.v_head, by_k.v_image, &blocks);
    if (!blocks) return hipSuccess;
    return with_type(type, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        hipLaunchKernelGGL((attention_add_kernel<T>), dim3(blocks), dim3(kThreads), 0, s, by_q, by_k, q, k, v.to);
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

// How a call is cut: a model of times in us.  Tiles take what the matrix products take at the rate that the kernels reach on a full card (1e15 operations a second,
// f32 1.2e14), for few rows what the memory takes (5 TB/s) and 1.6 us at least; a compute unit has its workgroups' tiles one after the other, and 4 us for the beginning and end
// of those that it has at a time.  Where parts differ (causal, keys' gradients beside queries'), the longest workgroup bounds the launch, and the compute units are not done at one time:
// 0.4 of the longest behind their average.  The join is a launch (5 us) that reads what the splits write (6 TB/s, both).
namespace {

struct CutModel {
    AttnCut cut;
    int64_t tiles, blocks;
    double share;    // of the tiles that a part sees on average where causal: of Lq x Lk, all but a triangle
    double tile_us, least_us, part_us;
    int at_once;     // workgroups on a compute unit
    int num_cu;
    CutModel(const qrm_attention_desc &d, int width, int kind, int cus) : cut{}, num_cu(cus)
    {
        const int size = type_bytes(d.type), w = cut.width = attn_width(size, width);
        const bool keys = kind == ATTN_DKV;
        const int64_t group = d.heads / d.kv_heads, columns = keys ? d.Lk : d.Lq * group, others = keys ? d.Lq : d.Lk;
        cut.kind = kind == ATTN_FORWARD && columns <= kAttnFew ? ATTN_FEW : kind;
        const bool few = cut.kind == ATTN_FEW;
        const AttnShape h = cut.shape = attn_shape(size, w, cut.kind);
        cut.parts = (int)((columns + h.rows() - 1) / h.rows());
        tiles = std::max<int64_t>(1, (others + h.tile - 1) / h.tile * (keys ? group : 1));
        blocks = d.N * d.kv_heads * cut.parts;
        const double lq = (double)d.Lq, lk = (double)d.Lk, seen = std::min(lq, lk);
        share = !d.causal || few || seen == 0.0 ? 1.0 : seen * (lk - 0.5 * seen) / (lq * lk);
        const double products = kind == ATTN_FORWARD ? 2.0 : kind == ATTN_DQ ? 3.0 : 4.0, rate = (size == 2 ? 1e9 : 1.2e8) / num_cu;
        tile_us = std::max(products * 2.0 * h.rows() * h.tile * w / rate, few ? 2.0 * h.tile * w * size / (5e6 / num_cu) : 0.0);
        least_us = few ? 1.6 : 1.1 * tile_us;
        part_us = (keys ? 2.0 : 1.0) * blocks * h.rows() * w * 8.0 / 6e6;
        at_once = std::max(1, std::min(h.occupancy * 4 / h.waves, (160 << 10) / (h.buffers * 2 * h.tile * attn_pitch(w * size) + 1024)));
        split(1);
    }
    // n splits, or as many as its tiles make
    void split(int64_t n)
    {
        n = std::min(n, tiles);
        cut.per = (int)((tiles + n - 1) / n);
        cut.splits = (int)((tiles + cut.per - 1) / cut.per);
    }
    double workgroups() const { return blocks * (share < 1.0 ? std::max(1.0, cut.splits * share + 0.5) : (double)cut.splits); }
    double longest() const { return cut.per * least_us; }
    double work() const { return blocks * tiles * share * tile_us / num_cu; }
    double join() const { return cut.splits > 1 ? part_us * cut.splits * share : 0.0; }
};
constexpr int kSplits[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64};

} // namespace

// Measured, us, by number of splits (the rule's in brackets): one head of 512, bf16, 4 x 1024 rows 1 74, 2 51, 3 42, [4 39], 6 39, 8 41; 4 x 4096 rows 1 254, [2 164], 3 206, 4 183; 16 heads of
// 128, 4 key heads, causal, 2 x 8192 rows [1 511], 2 645; 16 single tokens of 32 heads over up to 8191 rows of 4: 1 167, 4 49, 6 38, [8 34], 12 34; f32, 6 heads of 60, 3 x 2257 rows 1 298,
// 2 235, [3 211], 4 237.
AttnCut plan_attention(const qrm_attention_desc &d, int width, int num_cu)
{
    CutModel m(d, width, ATTN_FORWARD, num_cu), best = m;
    double least = 0.0;
    for (int n : kSplits) {
        if (n > m.tiles) break;
        m.split(n);
        const double on_one = std::ceil(m.workgroups() / num_cu), work = m.share < 1.0 ? m.work() + 0.4 * m.longest() : on_one * m.cut.per * m.tile_us;
        const double us = std::max(work, m.longest()) + std::ceil(on_one / m.at_once) * 4.0 + (m.cut.splits > 1 ? 5.0 + m.join() : 0.0);
        if (n == 1 || us < least) least = us, best = m;
    }
    return best.cut;
}

// Both sides of a backward launch, whatever of it is wanted: a gradient's bits do not depend on the others.  Measured, us of the call, by splits of queries' / keys' side: 16 heads of 128, 4 key
// heads, 2 x 4096 causal rows 1/1 634, 1/2 498, 1/3 460, 1/4 466, [1/5 470], 2 % from the best; one head of 512, 4 x 1024 rows 1/1 109, 1/2 82, 1/3 85, [2/2 79], 2/3 92; f16, 5 x 777 rows over 1033, 8 heads of 96,
// 2 key heads 1/1 119, 1/2 74, [1/3 63], 1/4 67, 2/4 62.
void plan_attention_backward(const qrm_attention_desc &d, int width, int num_cu, AttnCut *by_q, AttnCut *by_k)
{
    CutModel q(d, width, ATTN_DQ, num_cu), k(d, width, ATTN_DKV, num_cu);
    double least = 0.0;
    bool any = false;
    for (int n : kSplits) {
        if (n > q.tiles) break;
        q.split(n);
        for (int m : kSplits) {
            if (m > k.tiles) break;
            k.split(m);
            const double work = q.work() + k.work(), longest = std::max(q.longest(), k.longest()), workgroups = q.workgroups() + k.workgroups();
            const double us = std::max(work + 0.4 * longest, longest) + std::ceil(workgroups / num_cu / std::min(q.at_once, k.at_once)) * 4.0 + (n > 1 || m > 1 ? 5.0 + q.join() + k.join() : 0.0);
            if (!any || us < least) least = us, any = true, *by_q = q.cut, *by_k = k.cut;
        }
    }
}

} // namespace qrm
