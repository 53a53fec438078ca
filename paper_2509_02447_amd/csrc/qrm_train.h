// Shared by the fine-tuning operators (group_norm.hip, adamw.hip, message_loss.hip, qrm_train.hip): element types, wide loads and
// stores, launchers.
#pragma once

#include <type_traits>

#include "qrm_internal.h"

namespace qrm {

typedef _Float16 f16_t;

// V neighbouring elements as one load or store of up to 16 bytes.  STREAM: past the caches, for what will not be read from them.
template <typename T, int V> struct alignas(sizeof(T) * V) Pack {
    T e[V];
};
template <int BYTES> struct Raw {
    typedef uint32_t type __attribute__((ext_vector_type(BYTES / 4)));
};
template <> struct Raw<4> { typedef uint32_t type; };
template <> struct Raw<2> { typedef uint16_t type; };
template <typename T, int V, bool STREAM = false> __device__ __forceinline__ Pack<T, V> load_pack(const T *p)
{
    typedef typename Raw<sizeof(T) * V>::type R;
    typedef Pack<T, V> P;
    return __builtin_bit_cast(P, STREAM ? __builtin_nontemporal_load((const R *)p) : *(const R *)p);
}
template <typename T, int V, bool STREAM = false> __device__ __forceinline__ void store_pack(T *p, const Pack<T, V> &v)
{
    typedef typename Raw<sizeof(T) * V>::type R;
    if (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(R, v), (R *)p);
    else *(R *)p = __builtin_bit_cast(R, v);
}

// The same as the 32-bit registers that they were loaded into: elements are widened where they are used and, behind a pin(), widened again
// there instead of being kept as 32-bit numbers in between.
template <typename T, int V> struct Words {
    static constexpr int N = (V * (int)sizeof(T) + 3) / 4;
    uint32_t w[N];
    __device__ __forceinline__ void pin()
    {
#pragma unroll
        for (int i = 0; i < N; ++i) asm volatile("" : "+v"(w[i]));
    }
    __device__ __forceinline__ float get(int v) const
    {
        if constexpr (sizeof(T) == 4) {
            return __uint_as_float(w[v]);
        } else if constexpr (std::is_same<T, bf16_t>::value) {
            return __uint_as_float(v & 1 ? w[v / 2] & 0xffff0000u : w[v / 2] << 16);
        } else {
            return (float)__builtin_bit_cast(f16_t, (uint16_t)(w[v / 2] >> (v & 1 ? 16 : 0)));
        }
    }
    __device__ __forceinline__ void set(const float (&f)[V])
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int v = 0; v < V; ++v) w[v] = __float_as_uint(f[v]);
        } else if constexpr (V == 1) {
            w[0] = __builtin_bit_cast(uint16_t, (T)f[0]);
        } else {
            typedef T pair __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int v = 0; v < V; v += 2) w[v / 2] = __builtin_bit_cast(uint32_t, (pair){(T)f[v], (T)f[v + 1]});
        }
    }
};
template <typename T, int V> __device__ __forceinline__ Words<T, V> load_words(const T *p)
{
    Words<T, V> r;
    if constexpr (V * sizeof(T) == 2) {
        r.w[0] = *(const uint16_t *)p;
    } else {
        typedef uint32_t vec __attribute__((ext_vector_type(Words<T, V>::N)));
        const vec v = *(const vec *)p;
#pragma unroll
        for (int i = 0; i < Words<T, V>::N; ++i) r.w[i] = v[i];
    }
    return r;
}
// STREAM: past the caches, for what will not be read from them.
template <bool STREAM, typename T, int V> __device__ __forceinline__ void store_words(T *p, const Words<T, V> &r)
{
    if constexpr (V * sizeof(T) == 2) {
        *(uint16_t *)p = (uint16_t)r.w[0];
    } else {
        typedef uint32_t vec __attribute__((ext_vector_type(Words<T, V>::N)));
        vec v;
#pragma unroll
        for (int i = 0; i < Words<T, V>::N; ++i) v[i] = r.w[i];
        if (STREAM) __builtin_nontemporal_store(v, (vec *)p);
        else *(vec *)p = v;
    }
}

inline int type_bytes(int type) { return type == QRM_F32 ? 4 : 2; }

// Calls f with a null pointer of the element type.
template <typename F> auto with_type(int type, F &&f)
{
    return type == QRM_F32 ? f((float *)nullptr) : type == QRM_BF16 ? f((bf16_t *)nullptr) : f((f16_t *)nullptr);
}

// ---- group norm

constexpr int kNormThreads = 256, kNormMaxThreads = 1024;
// Pixels a thread holds in one launch: as many as the registers take, or few.
constexpr int norm_many(bool backward, int W) { return backward ? (W <= 2 ? 12 : 8) : W <= 2 ? 16 : 8; }
constexpr int kNormFew = 4;
// .. and walks down in the first of two launches: what it adds up in 32 bits stays short (norm_stats_kernel, norm_grad_sums_kernel).
constexpr int kNormRow = 2048;

// How a launch cuts a map: tiles of `ct` channels (whole groups, the last one narrower), of which a workgroup takes a chunk of one image's pixels.
struct NormCut {
    int ct, tiles, threads;
    int chunks; // workgroups to a tile of an image
    uint32_t blocks(int64_t N) const { return (uint32_t)(N * tiles * chunks); }
};
struct NormPlan {
    int V;             // channels that are read at once
    int W;             // sets of statistics to such a piece: one where V divides a group, the groups in it where groups divide V, else V
    NormCut first, second;
    bool whole;        // one launch (`first`): a workgroup holds a whole tile of an image, up to `pixels` pieces a thread
    int pixels;
    bool stream;       // outputs past the caches
    bool channels;     // sums of the channels go through the workspace
    size_t part_words; // of the chunks' groups in the workspace, before the channels' sums
    size_t bytes;      // of workspace
};
struct NormCall {
    qrm_group_norm_desc d; // strides filled in
    const void *x, *dy;
    const float *gamma, *beta;
    float *mean, *rstd;    // forward: outputs, may be null; backward: inputs
    void *y, *dx;
    float *dgamma, *dbeta;
};
// false: the pieces of a group are too many.  channels: dgamma or dbeta is wanted.
bool plan_norm(const qrm_group_norm_desc &d, int align_bytes, bool backward, bool channels, int num_cu, NormPlan *out);
hipError_t launch_norm_forward(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s);
hipError_t launch_norm_backward(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s);

// ---- AdamW

struct AdamwTensor { // device copy of a qrm_adamw_tensor
    int64_t n;
    void *p, *m, *v, *copy;
    float *m_scale, *v_scale;
    float weight_decay, lr_scale;
};
constexpr int kAdamwPiece = 4096;  // elements of a workgroup's piece
constexpr int kAdamwGrads = 448;   // gradients named to one launch (3.5 KiB of arguments)
struct AdamwStep {
    float beta1, rest1, beta2, rest2, eps, lr, rate, root; // rest = 1 - beta, rate = lr / (1 - beta1^step), root = 1 / sqrt(1 - beta2^step)
    const float *grad_scale;
};
struct AdamwTypes {
    int param, grad, copy, bits;
    bool stream; // a step passes more bytes than the caches hold
};
// Pieces first .. first + count - 1 of the plan, which belong to tensors t0 .. t0 + grads - 1.
hipError_t launch_adamw(const AdamwTypes &t, const AdamwTensor *tensors, const uint2 *pieces, uint32_t first, uint32_t count, uint32_t t0,
                        const void *const *grads, int n_grads, const AdamwStep &step, hipStream_t s);
hipError_t launch_unpack_moment(int moment, const void *codes, const float *scales, int64_t n, int out_type, void *out, hipStream_t s);

// ---- norm of the gradients

struct NormParts {
    double *sums;         // of the workgroups of all launches
    uint32_t *done;       // counters, all zero
    uint32_t first, total; // this launch's first one, all of them
    bool ends;            // this is the last launch
    double max_norm;
    const float *unscale; // or null
    float *norm, *scale;  // either may be null
};
constexpr int kScaleGrads = kAdamwGrads / 2; // gradients named to one launch that has outputs too
uint32_t norm_blocks(uint32_t pieces);
// Pieces and gradients as launch_adamw; no pieces: one workgroup.
hipError_t launch_grad_norm(int type, const AdamwTensor *tensors, const uint2 *pieces, uint32_t first, uint32_t count, uint32_t t0, const void *const *grads, int n_grads,
                            const NormParts &parts, hipStream_t s);
hipError_t launch_scale_grads(int type, const AdamwTensor *tensors, const uint2 *pieces, uint32_t first, uint32_t count, uint32_t t0, const void *const *grads, void *const *outs, int n_grads,
                              const float *scale, hipStream_t s);

// ---- attention

// Quotients by a number that a launch keeps, of numbers below 2^31: the high half of a product with ceil(2^(31 + s) / d), s = ceil(log2 d), which is exact for them; a
// division takes thirty instructions, and a workgroup begins with a dozen.
struct Quotient {
    uint32_t by, factor;
    int shift;
    Quotient() = default;
    explicit Quotient(uint32_t d) : by(d), factor(0), shift(0)
    {
        while (((uint64_t)1 << shift) < d) ++shift;
        if (shift) factor = (uint32_t)((((uint64_t)1 << (31 + shift)) + d - 1) / d);
    }
    __device__ __forceinline__ int of(int n) const { return shift ? (int)(__umulhi((uint32_t)n, factor) >> (shift - 1)) : n; }
};
struct AttnArgs { // of the kernels; strides in elements; rows of D elements lie on 16 bytes and are a multiple of them (launch_attention_copy)
    const void *q, *k, *v, *dy;
    void *o, *dq, *dk, *dv;
    float *lse;                        // [N,heads,Lq]
    const float *row_lse, *row_delta;  // backward, [N,heads,Lq]: minus log-sums over the scale (-inf: the row sees nothing), minus sums of dy o
    float *part, *part_sums;           // splits > 1: their results, and forward (raw score, sum about it) of each row (store_part)
    float *part_k, *part_v;
    const int32_t *q_len, *k_len;      // [N] or null
    int64_t q_row, q_head, q_image, k_row, k_head, k_image, v_row, v_head, v_image, o_row, o_head, o_image;
    int N, Lq, Lk, heads, kv_heads, group, D;
    int parts, splits, per;            // of the launch: tiles of the columns' rows, the most splits of the other side, and its tiles in one
    int columns, tile_shift;           // rows of a part, of a tile of the other side (2 to that)
    Quotient by_group, by_kv_heads, by_parts, by_blocks, by_per; // by_blocks: parts * splits
    float scale;
    bool causal;
};
// How a kernel cuts its work: columns of a wavefront (the matrix products' side), wavefronts of a workgroup, how many of them share a set of columns, rows of
// the other side in a tile, tiles in LDS, wavefronts to a SIMD that the registers are kept for.
// Tiles and wavefronts as measured, us (forward, bf16): one head of 512, 4 x 4096 rows, 16 columns in each of eight wavefronts with two tiles in LDS 164, two wavefronts to 32 columns 184 (two
// tiles) and 200 (one); rows of 64 and less in tiles of 64 keys or 32: f32 or bf16 over 4096 keys 170 and 179, over 77 keys 21 and 19.6: 64 for all
// lengths, for the long ones' sake.
struct AttnShape {
    int m, waves, share, tile, buffers, occupancy;
    constexpr int rows() const { return m * waves / share; }
};
enum { ATTN_FORWARD, ATTN_FEW, ATTN_DQ, ATTN_DKV }; // ATTN_FEW: forward with up to kAttnFew query rows to a key head
// (they fill no workgroup of four wavefronts: 16 single tokens of 8 heads to a key head 41 us with 32 columns to a wavefront, 38 with 16)
constexpr int kAttnFew = 32;
// Elements of a row that a kernel is made for.  (Half a row is whole pieces of 256 bytes where two wavefronts share columns: no 192 of f32.)
constexpr int attn_width(int size, int D) { return D <= 32 ? 32 : D <= 64 ? 64 : D <= 96 ? 96 : D <= 128 ? 128 : D <= 192 && size == 2 ? 192 : D <= 256 ? 256 : 512; }
constexpr int attn_pitch(int bytes) { return bytes <= 128 ? 128 : bytes <= 256 ? 256 : bytes <= 512 ? 512 : bytes <= 1024 ? 1024 : 2048; } // of a row in LDS
constexpr AttnShape attn_shape(int size, int width, int kind)
{
    const int bytes = attn_pitch(size * width);
    switch (kind) {
    case ATTN_FEW:
        return bytes <= 256 ? AttnShape{16, 1, 1, 32, 2, 2} : bytes == 512 ? AttnShape{16, 1, 1, 32, 2, 1} : AttnShape{16, 2, 2, 32, 1, 1};
    case ATTN_FORWARD:
        return bytes <= 128 ? AttnShape{32, 4, 1, 64, 2, 4} : bytes == 256 ? AttnShape{32, 4, 1, 64, 2, 2} : bytes == 512 ? AttnShape{32, 4, 1, 32, 2, 2} : bytes == 1024 ? AttnShape{size == 2 ? 16 : 32, 8, size == 2 ? 1 : 2, 32, size == 2 ? 2 : 1, 2} : AttnShape{16, 8, 2, 32, 1, 2};
    case ATTN_DQ:
        return bytes <= 256 ? AttnShape{32, 4, 1, 64, 2, 2} : bytes == 512 ? AttnShape{16, 4, 1, 32, 2, 2} : AttnShape{16, 8, 2, 32, bytes == 1024 ? 2 : 1, 2};
    default:
        return bytes <= 128 ? AttnShape{32, 4, 1, 64, 2, 2} : bytes == 256 ? AttnShape{32, 4, 1, 32, 2, 2} : bytes == 512 ? AttnShape{16, 4, 1, 32, 2, 2} : AttnShape{16, 8, 2, 32, bytes == 1024 ? 2 : 1, 2};
    }
}
// The registers hold the sums of dk and dv beside the keys and values, or they are two launches (f32 rows of 512 elements: 4 x 1024 of one head, the whole call 407 us; 449 while
// addresses that were kept from tile to tile pushed 48 registers into scratch).
constexpr bool attn_dk_dv_at_once(int size, int width) { return attn_pitch(size * width) <= 1024; }
struct AttnRows { // where rows [N,L,heads,D] lie
    int64_t row, head, image;
};
struct AttnCut {
    int kind, parts, splits, per, width; // width: of the kernel
    AttnShape shape;
    // bytes that wait for the other splits': results, or forward their rows' sums
    size_t part_bytes(const qrm_attention_desc &d) const { return splits > 1 ? (size_t)splits * d.N * d.kv_heads * parts * shape.rows() * width * 4 : 0; }
    size_t sums_bytes(const qrm_attention_desc &d) const { return splits > 1 ? (size_t)splits * d.N * d.kv_heads * parts * shape.rows() * 8 : 0; }
    // threads of the launch (workgroups in eights), and of what joins one of its results: a launch has less than 2^32
    double threads(const qrm_attention_desc &d) const { return ((double)d.N * d.kv_heads * parts * splits + 8) * shape.waves * 64; }
    double join_threads(const qrm_attention_desc &d) const { return splits > 1 ? (double)d.N * d.kv_heads * parts * shape.rows() * width / 8 + 256 : 0.0; }
};
// A part's splits: a workgroup walks down `per` tiles at most; a part of no more is written at once, the results of others are joined.  Both here and there
// as many as are walked down at all: tiles of an image's length, not of Lk.
struct AttnSplit {
    int count, from, to;
};
__device__ __forceinline__ AttnSplit attn_split(const AttnArgs &a, int tiles, int which)
{
    if (tiles <= a.per) return AttnSplit{1, 0, tiles};
    const int count = a.by_per.of(tiles + a.per - 1), each = (tiles + count - 1) / count;
    return AttnSplit{count, which * each, min(tiles, (which + 1) * each)};
}
__device__ __forceinline__ int attn_length(const int32_t *lens, int n, int all) { return lens ? max(0, min(lens[n], all)) : all; }
// Forward, probabilities of f16 are taken times two to that (attention_kernel).
constexpr float attn_lift(bool f16) { return f16 ? 11.f : 0.f; }
// The log-sum of a row whose probabilities about the raw score `top`, lifted, have the sum `sum`.  Past 32 bits' largest, up or down, it is no number: -inf is the
// log-sum of a row that sees nothing.
__device__ __forceinline__ float attn_log_sum(float top, float scale, float sum, float lift)
{
    const float lse = __builtin_fmaf(top, scale, (__builtin_amdgcn_logf(sum) - lift) * 0.693147180559945309f);
    return fabsf(lse) < INFINITY ? lse : NAN;
}
// Query rows are counted position by position, the heads of a group side by side.
__device__ __forceinline__ int attn_position(const AttnArgs &a, int row) { return a.by_group.of(row); }
// Tiles of keys that any of a part's query rows sees; tiles of a head's queries (behind `skip`) that see any of a part's keys.
__device__ __forceinline__ int attn_key_tiles(const AttnArgs &a, int q_len, int k_len, int part)
{
    const int first = attn_position(a, part * a.columns);
    if (first >= q_len) return 0;
    const int last = min(attn_position(a, part * a.columns + a.columns - 1), q_len - 1);
    return ((a.causal ? max(0, min(k_len, last + k_len - q_len + 1)) : k_len) + (1 << a.tile_shift) - 1) >> a.tile_shift;
}
__device__ __forceinline__ int attn_query_tiles(const AttnArgs &a, int q_len, int k_len, int part, int *skip)
{
    const int base = part * a.columns;
    *skip = a.causal ? max(0, base - (k_len - q_len)) >> a.tile_shift : 0;
    return base < k_len ? max(0, ((q_len + (1 << a.tile_shift) - 1) >> a.tile_shift) - *skip) : 0;
}
// width: D rounded up to 16 bytes.
AttnCut plan_attention(const qrm_attention_desc &d, int width, int num_cu);
void plan_attention_backward(const qrm_attention_desc &d, int width, int num_cu, AttnCut *by_q, AttnCut *by_k);
hipError_t launch_attention(int type, int kind, const AttnArgs &a, hipStream_t s); // forward
hipError_t launch_attention_backward(int type, const AttnArgs &by_q, const AttnArgs &by_k, hipStream_t s); // dq, dk and dv, those that are not null
// Backward, before all else: row_lse and row_delta of lse, o and dy.
hipError_t launch_attention_rows(const qrm_attention_desc &d, const void *o, const void *dy, const float *lse, const int32_t *q_len, float *row_lse, float *row_delta, hipStream_t s);
// Behind launches with splits: what they have left, into o and lse, or into dq, dk and dv (those that are not null and were split).
hipError_t launch_attention_join(int type, const AttnArgs &a, const AttnCut &cut, hipStream_t s);
hipError_t launch_attention_add(int type, const AttnArgs &by_q, const AttnCut &cut_q, const AttnArgs &by_k, const AttnCut &cut_k, hipStream_t s);
// Rows of any alignment into rows [N,heads,L,wide] that the kernels take, or (out) back.
hipError_t launch_attention_copy(int type, bool out, const AttnRows &r, void *there, void *here, int64_t N, int64_t L, int heads, int D, int wide, hipStream_t s);

// ---- message loss

struct LossCall {
    const float *logits;
    const uint8_t *target;
    int64_t target_stride; // 0: one target for all images
    int64_t N;
    int n_bits, m, n, t;   // without a code: symbols of one bit
    float weight;
    float *loss, *grad;
    int32_t *bit_errors, *symbol_errors;
};
int64_t loss_blocks(int64_t N, int n);
hipError_t launch_message_loss(const LossCall &c, double *partial, uint32_t *done, hipStream_t s);

} // namespace qrm
