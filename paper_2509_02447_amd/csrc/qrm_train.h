// Shared by the fine-tuning operators (group_norm.hip, adamw.hip, message_loss.hip, qrm_train.hip): element types, wide loads and
// stores, launchers.
#pragma once

#include "qrm_internal.h"

namespace qrm {

typedef _Float16 f16_t;

// V neighbouring elements as one load or store of up to 16 bytes.
template <typename T, int V> struct alignas(sizeof(T) * V) Pack {
    T e[V];
};
template <typename T, int V> __device__ __forceinline__ Pack<T, V> load_pack(const T *p) { return *(const Pack<T, V> *)p; }
template <typename T, int V> __device__ __forceinline__ void store_pack(T *p, const Pack<T, V> &v) { *(Pack<T, V> *)p = v; }

inline int type_bytes(int type) { return type == QRM_F32 ? 4 : 2; }

// Calls f with a null pointer of the element type.
template <typename F> auto with_type(int type, F &&f)
{
    return type == QRM_F32 ? f((float *)nullptr) : type == QRM_BF16 ? f((bf16_t *)nullptr) : f((f16_t *)nullptr);
}

// ---- group norm

// How a map is cut: tiles of `ct` channels (whole groups, the last one narrower), of which a workgroup takes `rows` pixels of one
// image; V channels are read at once.
struct NormPlan {
    int V, ct, tiles, threads;
    int64_t rows;
    int chunks;      // workgroups to a tile of an image
    bool uniform;    // V divides a group: the channels read at once belong to one group
    size_t bytes;    // of workspace
};
struct NormCall {
    qrm_group_norm_desc d; // strides filled in
    const void *x, *dy;
    const float *gamma, *beta;
    float *mean, *rstd;    // forward: outputs, may be null; backward: inputs
    void *y, *dx;
    float *dgamma, *dbeta;
};
// false: the pieces of a group are too many
bool plan_norm(const qrm_group_norm_desc &d, int align_bytes, bool backward, int num_cu, NormPlan *out);
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
};
// Pieces first .. first + count - 1 of the plan, which belong to tensors t0 .. t0 + grads - 1.
hipError_t launch_adamw(const AdamwTypes &t, const AdamwTensor *tensors, const uint2 *pieces, uint32_t first, uint32_t count, uint32_t t0,
                        const void *const *grads, int n_grads, const AdamwStep &step, hipStream_t s);
hipError_t launch_unpack_moment(int moment, const void *codes, const float *scales, int64_t n, int out_type, void *out, int num_cu, hipStream_t s);

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
hipError_t launch_message_loss(const LossCall &c, double *partial, hipStream_t s);

} // namespace qrm
