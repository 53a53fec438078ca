// Entry points of the fine-tuning operators (include/qrm.h): argument checks, plans and workspaces.  Host code only.
#include "qrm_train.h"

#include <math.h>
#include <stdio.h>

#include <new>
#include <vector>

#include "qrm_ctx.h"

using namespace qrm;

struct qrm_adamw {
    int device = 0;
    AdamwTypes types{};
    void *memory = nullptr;            // tensors, then pieces
    const AdamwTensor *tensors = nullptr;
    const uint2 *pieces = nullptr;     // (tensor, piece of it), tensor after tensor
    std::vector<uint32_t> first_piece; // [n_tensors + 1]
};

namespace {

bool known_type(int t) { return t == QRM_F32 || t == QRM_BF16 || t == QRM_F16; }
bool aligned_to(const void *p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// The largest power of two up to 16 that divides all addresses.
int common_alignment(std::initializer_list<const void *> list)
{
    uintptr_t bits = 16;
    for (const void *p : list) bits |= (uintptr_t)p;
    return (int)(bits & (~bits + 1));
}

// Fills in dense strides and checks what both directions share.
qrm_status check_norm(qrm_ctx *c, const qrm_group_norm_desc *desc, qrm_group_norm_desc *d)
{
    if (!desc) return fail(c, QRM_E_INVALID, "desc is NULL");
    *d = *desc;
    if (d->N < 0 || d->P < 1) return fail(c, QRM_E_INVALID, "need N >= 0 and P >= 1");
    if (d->C < 1 || d->groups < 1 || d->C % d->groups) return fail(c, QRM_E_INVALID, "groups must divide C");
    if (!known_type(d->type)) return fail(c, QRM_E_INVALID, "unknown type");
    if (d->act != QRM_ACT_NONE && d->act != QRM_ACT_RELU && d->act != QRM_ACT_SILU) return fail(c, QRM_E_INVALID, "unknown activation");
    if (!(d->eps > 0.f) || !std::isfinite(d->eps)) return fail(c, QRM_E_INVALID, "eps must be above zero");
    if (d->C > 65536 || d->N > INT32_MAX || d->P > INT32_MAX) return fail(c, QRM_E_UNSUPPORTED, "C up to 65536, N and P below 2^31");
    constexpr int64_t far = (int64_t)1 << 46; // (addresses stay in 64 bits)
    for (int64_t *st : {&d->x_pixel, &d->y_pixel}) {
        if (!*st) *st = d->C;
        if (*st < d->C || *st > far / d->P) return fail(c, QRM_E_INVALID, "a pixel's stride is under C or out of range");
    }
    const int64_t pixel[2] = {d->x_pixel, d->y_pixel};
    int64_t *image[2] = {&d->x_image, &d->y_image};
    for (int i = 0; i < 2; ++i) {
        if (!*image[i]) *image[i] = d->P * pixel[i];
        if (*image[i] < (d->P - 1) * pixel[i] + d->C) return fail(c, QRM_E_INVALID, "images overlap: an image's stride is too short");
        if (d->N > 1 && *image[i] > far / d->N * 64) return fail(c, QRM_E_INVALID, "an image's stride is out of range");
    }
    return QRM_OK;
}

// An output in place of an input has to have its strides: otherwise it falls on pixels that are still to be read.
bool same_places(const qrm_group_norm_desc &d)
{
    return (d.P == 1 || d.x_pixel == d.y_pixel) && (d.N <= 1 || d.x_image == d.y_image);
}

qrm_status start(qrm_ctx *c)
{
    hipError_t e = hipSetDevice(c->device);
    return e == hipSuccess ? QRM_OK : hip_fail(c, e, "hipSetDevice");
}

qrm_status plan(qrm_ctx *c, const qrm_group_norm_desc &d, int align, bool backward, bool channels, NormPlan *p)
{
    if (!plan_norm(d, align, backward, channels, c->num_cu, p))
        return fail(c, QRM_E_UNSUPPORTED, "a group has more than 1024 pieces: its channels over their common divisor with the elements that are read at once");
    // (a launch has less than 2^32 threads; those behind the tiles, of the channels, are under 2^24)
    auto fits = [&](const NormCut &cut) { return ((double)d.N * cut.tiles * cut.chunks + 8192.0) * cut.threads < 4294967296.0; };
    if (!fits(p->first) || (!p->whole && !fits(p->second))) return fail(c, QRM_E_UNSUPPORTED, "the tiles of all images need 2^32 threads and more");
    return QRM_OK;
}

} // namespace

extern "C" {

qrm_status qrm_group_norm(qrm_ctx *c, const qrm_group_norm_desc *desc, const void *d_x, const float *d_gamma, const float *d_beta, void *d_y,
                          float *d_mean, float *d_rstd, void *stream)
{
    if (!c) return QRM_E_INVALID;
    NormCall call{};
    qrm_status st = check_norm(c, desc, &call.d);
    if (st != QRM_OK) return st;
    if (!d_mean != !d_rstd) return fail(c, QRM_E_INVALID, "d_mean and d_rstd go together");
    if (call.d.N == 0) return QRM_OK;
    if (!d_x || !d_y) return fail(c, QRM_E_INVALID, "d_x / d_y is NULL");
    if (d_x == d_y && !same_places(call.d)) return fail(c, QRM_E_INVALID, "d_y is d_x, with other strides");
    const int align = common_alignment({d_x, d_y});
    if (align < type_bytes(call.d.type) || !aligned_to(d_gamma, 4) || !aligned_to(d_beta, 4) || !aligned_to(d_mean, 4) || !aligned_to(d_rstd, 4))
        return fail(c, QRM_E_INVALID, "a pointer is not aligned to its elements");
    NormPlan p;
    if ((st = plan(c, call.d, align, false, false, &p)) != QRM_OK || (st = start(c)) != QRM_OK) return st;
    call.x = d_x; call.y = d_y; call.gamma = d_gamma; call.beta = d_beta; call.mean = d_mean; call.rstd = d_rstd;
    QrmSlot *slot = nullptr;
    if (p.bytes && (st = get_slot(c, (hipStream_t)stream, p.bytes, &slot)) != QRM_OK) return st;
    hipError_t e = launch_norm_forward(call, p, slot ? slot->ws : nullptr, (hipStream_t)stream);
    if (slot) st = slot_done(c, slot, (hipStream_t)stream, true);
    return e == hipSuccess ? st : hip_fail(c, e, "group_norm launch");
}

qrm_status qrm_group_norm_backward(qrm_ctx *c, const qrm_group_norm_desc *desc, const void *d_x, const void *d_dy, const float *d_gamma,
                                   const float *d_beta, const float *d_mean, const float *d_rstd, void *d_dx, float *d_dgamma, float *d_dbeta,
                                   void *stream)
{
    if (!c) return QRM_E_INVALID;
    NormCall call{};
    qrm_status st = check_norm(c, desc, &call.d);
    if (st != QRM_OK) return st;
    const bool none = call.d.N == 0;
    if (!none && (!d_x || !d_dy || !d_mean || !d_rstd)) return fail(c, QRM_E_INVALID, "d_x / d_dy / d_mean / d_rstd is NULL");
    if (!d_dx && !d_dgamma && !d_dbeta) return fail(c, QRM_E_INVALID, "no output is asked for");
    if (!none && d_dx == d_dy && !same_places(call.d)) return fail(c, QRM_E_INVALID, "d_dx is d_dy, with other strides");
    const int align = common_alignment({d_x, d_dy, d_dx});
    if (align < type_bytes(call.d.type) || !aligned_to(d_gamma, 4) || !aligned_to(d_beta, 4) || !aligned_to(d_mean, 4) || !aligned_to(d_rstd, 4) ||
        !aligned_to(d_dgamma, 4) || !aligned_to(d_dbeta, 4))
        return fail(c, QRM_E_INVALID, "a pointer is not aligned to its elements");
    call.x = d_x; call.dy = d_dy; call.gamma = d_gamma; call.beta = d_beta; call.mean = (float *)d_mean; call.rstd = (float *)d_rstd;
    call.dx = none ? nullptr : d_dx; call.dgamma = d_dgamma; call.dbeta = d_dbeta;
    NormPlan p{};
    if (none) {
        if (!d_dgamma && !d_dbeta) return QRM_OK;
        if ((st = start(c)) != QRM_OK) return st;
        hipError_t e = launch_norm_backward(call, p, nullptr, (hipStream_t)stream);
        return e == hipSuccess ? QRM_OK : hip_fail(c, e, "group_norm_backward launch");
    }
    if ((st = plan(c, call.d, align, true, d_dgamma || d_dbeta, &p)) != QRM_OK || (st = start(c)) != QRM_OK) return st;
    QrmSlot *slot = nullptr;
    if (p.bytes && (st = get_slot(c, (hipStream_t)stream, p.bytes, &slot)) != QRM_OK) return st;
    hipError_t e = launch_norm_backward(call, p, slot ? slot->ws : nullptr, (hipStream_t)stream);
    if (slot) st = slot_done(c, slot, (hipStream_t)stream, true);
    return e == hipSuccess ? st : hip_fail(c, e, "group_norm_backward launch");
}

qrm_status qrm_adamw_create(qrm_ctx *c, const qrm_adamw_desc *desc, const qrm_adamw_tensor *h_tensors, qrm_adamw **out)
{
    if (!c) return QRM_E_INVALID;
    if (!out) return fail(c, QRM_E_INVALID, "out is NULL");
    *out = nullptr;
    if (!desc || desc->n_tensors < 0 || (desc->n_tensors && !h_tensors)) return fail(c, QRM_E_INVALID, "desc / h_tensors is NULL or n_tensors < 0");
    if (!known_type(desc->param_type) || !known_type(desc->grad_type)) return fail(c, QRM_E_INVALID, "unknown type");
    if (desc->state_bits != 8 && desc->state_bits != 32) return fail(c, QRM_E_INVALID, "state_bits must be 8 or 32");
    const size_t pb = type_bytes(desc->param_type), mb = desc->state_bits / 8;
    const int n = desc->n_tensors;
    std::vector<AdamwTensor> tensors;
    std::vector<uint2> pieces;
    std::vector<uint32_t> first;
    uint64_t elements = 0;
    try {
        uint64_t total = 0;
        for (int i = 0; i < n; ++i) {
            const qrm_adamw_tensor &t = h_tensors[i];
            const bool eight = desc->state_bits == 8;
            if (t.n < 0) return fail(c, QRM_E_INVALID, "a tensor has n < 0");
            if (t.n && (!t.d_param || !t.d_m || !t.d_v || (eight && (!t.d_m_scale || !t.d_v_scale)))) return fail(c, QRM_E_INVALID, "a tensor's pointer is NULL");
            if (!aligned_to(t.d_param, pb) || !aligned_to(t.d_m, mb) || !aligned_to(t.d_v, mb) || !aligned_to(t.d_m_scale, 4) || !aligned_to(t.d_v_scale, 4) ||
                !aligned_to(t.d_copy, 2))
                return fail(c, QRM_E_INVALID, "a pointer is not aligned to its elements");
            if (t.d_copy && (desc->param_type != QRM_F32 || (desc->copy_type != QRM_BF16 && desc->copy_type != QRM_F16)))
                return fail(c, QRM_E_INVALID, "a copy is of 16 bits, beside f32 parameters");
            if (!(t.weight_decay >= 0.f) || !(t.lr_scale >= 0.f) || !std::isfinite(t.weight_decay) || !std::isfinite(t.lr_scale))
                return fail(c, QRM_E_INVALID, "weight_decay and lr_scale must be finite and not negative");
            total += ((uint64_t)t.n + kAdamwPiece - 1) / kAdamwPiece;
            elements += (uint64_t)t.n;
            if (total >= (1u << 24)) return fail(c, QRM_E_UNSUPPORTED, "2^24 and more pieces of 4096 elements"); // (a launch has less than 2^32 threads)
        }
        tensors.reserve(n);
        pieces.reserve(total);
        first.reserve(n + 1);
        for (int i = 0; i < n; ++i) {
            const qrm_adamw_tensor &t = h_tensors[i];
            tensors.push_back(AdamwTensor{t.n, t.d_param, t.d_m, t.d_v, t.d_copy, t.d_m_scale, t.d_v_scale, t.weight_decay, t.lr_scale});
            first.push_back((uint32_t)pieces.size());
            const uint32_t count = (uint32_t)((t.n + kAdamwPiece - 1) / kAdamwPiece);
            for (uint32_t k = 0; k < count; ++k) pieces.push_back(make_uint2(i, k));
        }
        first.push_back((uint32_t)pieces.size());
    } catch (const std::bad_alloc &) {
        return fail(c, QRM_E_NOMEM, "no host memory for the plan");
    }
    qrm_status st = start(c);
    if (st != QRM_OK) return st;
    qrm_adamw *o = new (std::nothrow) qrm_adamw();
    if (!o) return fail(c, QRM_E_NOMEM, "no host memory for the plan");
    o->device = c->device;
    // Past the caches (8-bit moments excepted) where a step passes more than the memory-side cache holds (256 MiB): the next step finds nothing of it there.  50
    // million parameters with 16-bit gradients and a copy 278 us without, 266 with, with 8-bit moments 151 and 144; 200 million in 32 bits 1107 and 1053.
    const uint64_t each = 2 * pb + type_bytes(desc->grad_type) + 4 * mb; // bytes an element
    o->types = AdamwTypes{desc->param_type, desc->grad_type, desc->copy_type, desc->state_bits, elements * each > ((uint64_t)256 << 20)};
    o->first_piece = std::move(first);
    if (!pieces.empty()) {
        const size_t at = (tensors.size() * sizeof(AdamwTensor) + 255) / 256 * 256;
        hipError_t e = hipMalloc(&o->memory, at + pieces.size() * sizeof(uint2));
        if (e != hipSuccess) {
            (void)hipGetLastError();
            delete o;
            return fail(c, QRM_E_NOMEM, "no device memory for the plan");
        }
        e = hipMemcpy(o->memory, tensors.data(), tensors.size() * sizeof(AdamwTensor), hipMemcpyHostToDevice);
        if (e == hipSuccess) e = hipMemcpy((uint8_t *)o->memory + at, pieces.data(), pieces.size() * sizeof(uint2), hipMemcpyHostToDevice);
        if (e != hipSuccess) {
            (void)hipFree(o->memory);
            delete o;
            return hip_fail(c, e, "hipMemcpy(plan)");
        }
        o->tensors = (const AdamwTensor *)o->memory;
        o->pieces = (const uint2 *)((uint8_t *)o->memory + at);
    }
    *out = o;
    return QRM_OK;
}

void qrm_adamw_destroy(qrm_adamw *o)
{
    if (!o) return;
    if (o->memory) {
        (void)hipSetDevice(o->device);
        (void)hipDeviceSynchronize();
        (void)hipFree(o->memory);
    }
    delete o;
}

qrm_status qrm_adamw_step(qrm_ctx *c, qrm_adamw *o, const void *const *h_grads, int64_t step, double lr, double beta1, double beta2, double eps,
                          const float *d_grad_scale, void *stream)
{
    if (!c) return QRM_E_INVALID;
    if (!o) return fail(c, QRM_E_INVALID, "opt is NULL");
    if (o->device != c->device) return fail(c, QRM_E_INVALID, "the plan belongs to another device");
    if (step < 1) return fail(c, QRM_E_INVALID, "step counts from 1");
    if (!(lr >= 0.0) || !(eps >= 0.0) || !std::isfinite((float)lr) || !std::isfinite((float)eps)) return fail(c, QRM_E_INVALID, "lr and eps must be finite and not negative");
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0)) return fail(c, QRM_E_INVALID, "beta1 and beta2 must be in [0, 1)");
    if (!aligned_to(d_grad_scale, 4)) return fail(c, QRM_E_INVALID, "a pointer is not aligned to its elements");
    const int n = (int)o->first_piece.size() - 1;
    if (n <= 0) return QRM_OK;
    if (!h_grads) return fail(c, QRM_E_INVALID, "h_grads is NULL");
    const size_t gb = type_bytes(o->types.grad);
    for (int i = 0; i < n; ++i)
        if (!aligned_to(h_grads[i], gb)) return fail(c, QRM_E_INVALID, "a pointer is not aligned to its elements");
    qrm_status st = start(c);
    if (st != QRM_OK) return st;
    // (1 - beta from the caller's 64 bits: from a beta of 32 it would be off by 1e-5)
    AdamwStep s{(float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps, (float)lr, (float)(lr / (1.0 - pow(beta1, (double)step))),
                (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step))), d_grad_scale};
    for (int i = 0; i < n; i += kAdamwGrads) {
        const int count = n - i < kAdamwGrads ? n - i : kAdamwGrads;
        const uint32_t from = o->first_piece[i], to = o->first_piece[i + count];
        if (from == to) continue;
        hipError_t e = launch_adamw(o->types, o->tensors, o->pieces, from, to - from, i, h_grads + i, count, s, (hipStream_t)stream);
        if (e != hipSuccess) {
            char what[64];
            snprintf(what, sizeof what, "adamw launch of tensor %d and those behind it", i);
            return hip_fail(c, e, what);
        }
    }
    return QRM_OK;
}

qrm_status qrm_unpack_moment(qrm_ctx *c, int32_t moment, const void *d_codes, const float *d_scales, int64_t n, int32_t out_type, void *d_out, void *stream)
{
    if (!c) return QRM_E_INVALID;
    if (moment != 0 && moment != 1) return fail(c, QRM_E_INVALID, "moment is 0 or 1");
    if (n < 0) return fail(c, QRM_E_INVALID, "n < 0");
    if (out_type != QRM_F32 && out_type != QRM_BF16) return fail(c, QRM_E_INVALID, "values are f32 or bf16");
    if (n == 0) return QRM_OK;
    if (n >= (int64_t)1 << 36) return fail(c, QRM_E_UNSUPPORTED, "n of 2^36 and more"); // (a launch has less than 2^32 threads)
    if (!d_codes || !d_scales || !d_out) return fail(c, QRM_E_INVALID, "d_codes / d_scales / d_out is NULL");
    if (!aligned_to(d_scales, 4) || !aligned_to(d_out, type_bytes(out_type))) return fail(c, QRM_E_INVALID, "a pointer is not aligned to its elements");
    qrm_status st = start(c);
    if (st != QRM_OK) return st;
    hipError_t e = launch_unpack_moment(moment, d_codes, d_scales, n, out_type, d_out, (hipStream_t)stream);
    return e == hipSuccess ? QRM_OK : hip_fail(c, e, "unpack_moment launch");
}

qrm_status qrm_message_loss(qrm_ctx *c, const float *d_logits, const uint8_t *d_target, int64_t target_rows, int64_t N, int32_t n_bits, float rs_weight,
                            float *d_loss, float *d_grad, int32_t *d_bit_errors, int32_t *d_symbol_errors, void *stream)
{
    if (!c) return QRM_E_INVALID;
    if (N < 0) return fail(c, QRM_E_INVALID, "N < 0");
    if (n_bits < 1 || n_bits > 2040 || (c->has_rs && n_bits != c->rs.n * c->rs.m)) return fail(c, QRM_E_INVALID, "n_bits must be n * m, in 1 .. 2040");
    if (target_rows != 1 && target_rows != N) return fail(c, QRM_E_INVALID, "target_rows must be 1 or N");
    if (!(rs_weight >= 0.f) || !std::isfinite(rs_weight)) return fail(c, QRM_E_INVALID, "rs_weight must be finite and not negative");
    if (!c->has_rs && (rs_weight > 0.f || d_symbol_errors)) return fail(c, QRM_E_INVALID, "context has no Reed-Solomon code");
    if (!d_loss || (N && (!d_logits || !d_target))) return fail(c, QRM_E_INVALID, "d_logits / d_target / d_loss is NULL");
    if (!aligned_to(d_logits, 4) || !aligned_to(d_loss, 4) || !aligned_to(d_grad, 4) || !aligned_to(d_bit_errors, 4) || !aligned_to(d_symbol_errors, 4))
        return fail(c, QRM_E_INVALID, "a pointer is not aligned to its elements");
    if (N >= INT32_MAX / 64) return fail(c, QRM_E_UNSUPPORTED, "N of 2^31 / 64 and more");
    qrm_status st = start(c);
    if (st != QRM_OK) return st;
    LossCall call{d_logits, d_target, target_rows == 1 ? 0 : (int64_t)n_bits, N, n_bits, c->has_rs ? c->rs.m : 1, c->has_rs ? c->rs.n : n_bits,
                  c->has_rs ? c->rs.two_t / 2 : 0, rs_weight, d_loss, d_grad, d_bit_errors, d_symbol_errors};
    const int64_t blocks = loss_blocks(N, call.n);
    QrmSlot *slot = nullptr;
    if (blocks > 1 && ((st = get_slot(c, (hipStream_t)stream, (size_t)blocks * sizeof(double), &slot)) != QRM_OK ||
                       (st = get_counters(c, (hipStream_t)stream, slot)) != QRM_OK))
        return st;
    hipError_t e = launch_message_loss(call, slot ? (double *)slot->ws : nullptr, slot ? slot->counters : nullptr, (hipStream_t)stream);
    if (slot) st = slot_done(c, slot, (hipStream_t)stream, true);
    return e == hipSuccess ? st : hip_fail(c, e, "message_loss launch");
}

} // extern "C"
