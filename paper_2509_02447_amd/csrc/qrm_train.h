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
