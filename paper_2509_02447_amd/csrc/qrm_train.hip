// Entry points of the fine-tuning operators (include/qrm.h): argument checks, plans and workspaces.  Host code only.
#include "qrm_train.h"

#include <math.h>
#include <stdio.h>

#include <algorithm>
#include <functional>
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

// The gradients of a plan's tensors.
qrm_status check_grads(qrm_ctx *c, const qrm_adamw *o, const void *const *h_grads)
{
    const int n = (int)o->first_piece.size() - 1;
    if (n > 0 && !h_grads) return fail(c, QRM_E_INVALID, "h_grads is NULL");
    const size_t bytes = type_bytes(o->types.grad);
    for (int i = 0; i < n; ++i)
        if (!aligned_to(h_grads[i], bytes)) return fail(c, QRM_E_INVALID, "a pointer is not aligned to its elements");
    return QRM_OK;
}

// Each output of its own (an output's elements are written once: a gradient that two tensors share, scaled in place, would be scaled once or twice).
qrm_status check_outs(qrm_ctx *c, const qrm_adamw *o, void *const *h_outs)
{
    const int n = (int)o->first_piece.size() - 1;
    auto there = [&](int i) { return h_outs[i] && o->first_piece[i + 1] != o->first_piece[i]; };
    const void *last = nullptr;
    bool rising = true; // (one behind the other, as tensors mostly are: nothing to sort)
    for (int i = 0; i < n && rising; ++i)
        if (there(i)) rising = std::less<const void *>()(last, h_outs[i]), last = h_outs[i];
    if (rising) return QRM_OK;
    try {
        std::vector<const void *> all;
        all.reserve(n);
        for (int i = 0; i < n; ++i)
            if (there(i)) all.push_back(h_outs[i]);
        std::sort(all.begin(), all.end(), std::less<const void *>());
        if (std::adjacent_find(all.begin(), all.end()) != all.end()) return fail(c, QRM_E_INVALID, "two outputs are one");
    } catch (const std::bad_alloc &) {
        return fail(c, QRM_E_NOMEM, "no host memory for the outputs");
    }
    return QRM_OK;
}

constexpr double kLaunchThreads = 4294967296.0; // a launch has less
const char *const kTooManyRows = "the rows of all images need 2^32 threads and more";

// Where a tensor of an attention call lies: dense strides filled in; rows overlap nowhere.
qrm_status check_rows(qrm_ctx *c, AttnRows *r, int64_t N, int64_t L, int heads, int D)
{
    constexpr int64_t far = (int64_t)1 << 46; // (addresses stay in 64 bits)
    if (!r->head) r->head = D;
    if (!r->row) r->row = (int64_t)heads * D;
    if (!r->image) r->image = std::max<int64_t>(L, 1) * r->row;
    if (L <= 1) r->row = D; // (there is no next one)
    if (heads <= 1) r->head = D;
    if (N <= 1) r->image = D;
    std::pair<int64_t, int64_t> dims[3] = {{r->row, L}, {r->head, heads}, {r->image, N}};
    std::sort(dims, dims + 3);
    int64_t extent = D;
    for (auto &d : dims) {
        if (d.second <= 1) continue;
        if (d.first < extent) return fail(c, QRM_E_INVALID, "rows, heads or images overlap: a stride is too short");
        if (d.first > far / d.second) return fail(c, QRM_E_INVALID, "a stride is out of range");
        extent += d.first * (d.second - 1);
    }
    return QRM_OK;
}

struct AttnCheck {
    qrm_attention_desc d; // strides filled in
    AttnRows q, k, v, o;
    int wide;             // D rounded up to 16 bytes
};

qrm_status check_attention(qrm_ctx *c, const qrm_attention_desc *desc, AttnCheck *out)
{
    if (!desc) return fail(c, QRM_E_INVALID, "desc is NULL");
    qrm_attention_desc &d = out->d = *desc;
    if (d.N < 0 || d.Lq < 0 || d.Lk < 0) return fail(c, QRM_E_INVALID, "N, Lq and Lk must not be negative");
    if (d.heads < 1 || d.kv_heads < 1 || d.heads % d.kv_heads) return fail(c, QRM_E_INVALID, "kv_heads must divide heads");
    if (d.D < 1) return fail(c, QRM_E_INVALID, "D < 1");
    if (!known_type(d.type)) return fail(c, QRM_E_INVALID, "unknown type");
    if (d.causal != 0 && d.causal != 1) return fail(c, QRM_E_INVALID, "causal is 0 or 1");
    if (!(d.scale > 0.f) || !std::isfinite(d.scale)) return fail(c, QRM_E_INVALID, "scale must be above zero");
    if (d.scale < 0x1p-64f || d.scale > 0x1p64f) return fail(c, QRM_E_UNSUPPORTED, "scale outside 2^-64 .. 2^64");
    constexpr int64_t most = (int64_t)1 << 30;
    if (d.D > QRM_ATTENTION_MAX_D) return fail(c, QRM_E_UNSUPPORTED, "D above 512");
    if (d.N > most || d.Lq > most || d.Lk > most || d.Lq * d.heads > most) return fail(c, QRM_E_UNSUPPORTED, "N, Lk, or query rows of all heads of an image above 2^30");
    if (d.N * d.heads > most / 128) return fail(c, QRM_E_UNSUPPORTED, "heads of all images above 2^23");
    // (of the launches that take rows one by one: a thread has at least four elements, sixteen threads have a row)
    const double rows = (double)d.N * std::max((double)d.Lq * d.heads, (double)d.Lk * d.kv_heads);
    if (rows * ((d.D + 7) / 4) >= kLaunchThreads || rows * 16 >= kLaunchThreads) return fail(c, QRM_E_UNSUPPORTED, kTooManyRows);
    const int size = type_bytes(d.type), e = 16 / size;
    out->wide = (d.D + e - 1) / e * e;
    out->q = {d.q_row, d.q_head, d.q_image};
    out->k = {d.k_row, d.k_head, d.k_image};
    out->v = {d.v_row, d.v_head, d.v_image};
    out->o = {d.o_row, d.o_head, d.o_image};
    qrm_status st;
    for (AttnRows *r : {&out->q, &out->o})
        if ((st = check_rows(c, r, d.N, d.Lq, d.heads, d.D)) != QRM_OK) return st;
    for (AttnRows *r : {&out->k, &out->v})
        if ((st = check_rows(c, r, d.N, d.Lk, d.kv_heads, d.D)) != QRM_OK) return st;
    d.q_row = out->q.row, d.q_head = out->q.head, d.q_image = out->q.image;
    d.k_row = out->k.row, d.k_head = out->k.head, d.k_image = out->k.image;
    d.v_row = out->v.row, d.v_head = out->v.head, d.v_image = out->v.image;
    d.o_row = out->o.row, d.o_head = out->o.head, d.o_image = out->o.image;
    return QRM_OK;
}

// A tensor as the kernels see it: where it is, or rows of the workspace that it is copied to (and, an output, from) where it does not lie on 16 bytes.
struct AttnTensor {
    AttnRows rows;
    size_t at = 0; // in the workspace, where `copied`
    bool copied = false;
};

// Parts of a workspace, one behind the other.
struct Workspace {
    size_t bytes = 0;
    size_t take(size_t n)
    {
        const size_t at = bytes;
        bytes += (n + 255) / 256 * 256;
        return at;
    }
};

AttnTensor place(const AttnCheck &a, const AttnRows &r, int64_t L, int heads, std::initializer_list<const void *> list, int copies, Workspace *w)
{
    const int size = type_bytes(a.d.type), e = 16 / size;
    AttnTensor t;
    t.rows = r;
    // (the kernels multiply a tile's rows by their distance in 24 bits)
    t.copied = a.wide != a.d.D || common_alignment(list) < 16 || r.row % e || r.head % e || r.image % e || r.row * size >= (1 << 23);
    if (t.copied) {
        t.at = w->take((size_t)copies * a.d.N * heads * L * a.wide * size);
        t.rows = {a.wide, L * a.wide, heads * L * a.wide};
    }
    return t;
}

AttnArgs attention_args(const AttnCheck &a, const AttnTensor &q, const AttnTensor &k, const AttnTensor &v, const AttnTensor &o, const int32_t *q_len, const int32_t *k_len)
{
    const qrm_attention_desc &d = a.d;
    AttnArgs g{};
    g.q_len = q_len, g.k_len = k_len;
    g.q_row = q.rows.row, g.q_head = q.rows.head, g.q_image = q.rows.image;
    g.k_row = k.rows.row, g.k_head = k.rows.head, g.k_image = k.rows.image;
    g.v_row = v.rows.row, g.v_head = v.rows.head, g.v_image = v.rows.image;
    g.o_row = o.rows.row, g.o_head = o.rows.head, g.o_image = o.rows.image;
    g.N = (int)d.N, g.Lq = (int)d.Lq, g.Lk = (int)d.Lk, g.heads = d.heads, g.kv_heads = d.kv_heads, g.group = d.heads / d.kv_heads, g.D = a.wide;
    g.scale = d.scale, g.causal = d.causal != 0;
    return g;
}

void cut_to(AttnArgs *g, const AttnCut &cut)
{
    g->parts = cut.parts, g->splits = cut.splits, g->per = cut.per;
    g->columns = cut.shape.rows();
    for (g->tile_shift = 0; 1 << g->tile_shift < cut.shape.tile;) ++g->tile_shift;
    g->by_parts = Quotient(std::max(1, cut.parts)), g->by_blocks = Quotient(std::max(1, cut.parts * cut.splits)), g->by_per = Quotient(cut.per);
    g->by_group = Quotient(g->group), g->by_kv_heads = Quotient(g->kv_heads);
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
    qrm_status st = check_grads(c, o, h_grads);
    if (st != QRM_OK || (st = start(c)) != QRM_OK) return st;
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

qrm_status qrm_adamw_grad_norm(qrm_ctx *c, qrm_adamw *o, const void *const *h_grads, double max_norm, const float *d_unscale, float *d_norm, float *d_scale, void *stream)
{
    if (!c) return QRM_E_INVALID;
    if (!o) return fail(c, QRM_E_INVALID, "opt is NULL");
    if (o->device != c->device) return fail(c, QRM_E_INVALID, "the plan belongs to another device");
    if (!(max_norm > 0.0)) return fail(c, QRM_E_INVALID, "max_norm must be above zero");
    if (!d_norm && !d_scale) return fail(c, QRM_E_INVALID, "no output is asked for");
    if (d_norm == d_scale || (d_unscale && (d_unscale == d_norm || d_unscale == d_scale))) return fail(c, QRM_E_INVALID, "an output is an input or the other output");
    if (!aligned_to(d_unscale, 4) || !aligned_to(d_norm, 4) || !aligned_to(d_scale, 4)) return fail(c, QRM_E_INVALID, "a pointer is not aligned to its elements");
    qrm_status st = check_grads(c, o, h_grads);
    if (st != QRM_OK || (st = start(c)) != QRM_OK) return st;
    const int n = (int)o->first_piece.size() - 1;
    auto pieces = [&](int i) { return o->first_piece[std::min(n, i + kAdamwGrads)] - o->first_piece[i]; };
    NormParts parts{};
    for (int i = 0; i == 0 || i < n; i += kAdamwGrads) parts.total += n ? norm_blocks(pieces(i)) : 1;
    parts.max_norm = max_norm;
    parts.unscale = d_unscale, parts.norm = d_norm, parts.scale = d_scale;
    QrmSlot *slot = nullptr;
    const hipStream_t s = (hipStream_t)stream;
    if (parts.total > 1) {
        if ((st = get_slot(c, s, parts.total * sizeof(double), &slot)) != QRM_OK || (st = get_counters(c, s, slot)) != QRM_OK) return st;
        parts.sums = (double *)slot->ws;
        parts.done = slot->counters;
    }
    hipError_t e = hipSuccess;
    for (int i = 0; e == hipSuccess && (i == 0 || i < n); i += kAdamwGrads) {
        const uint32_t count = n ? pieces(i) : 0;
        parts.ends = i + kAdamwGrads >= n;
        e = launch_grad_norm(o->types.grad, o->tensors, o->pieces, n ? o->first_piece[i] : 0, count, i, n ? h_grads + i : nullptr, std::min(n - i, kAdamwGrads), parts, s);
        parts.first += norm_blocks(count);
    }
    if (slot) st = slot_done(c, slot, s, true);
    return e == hipSuccess ? st : hip_fail(c, e, "grad_norm launch");
}

qrm_status qrm_adamw_scale_grads(qrm_ctx *c, qrm_adamw *o, const void *const *h_grads, const float *d_scale, void *const *h_outs, void *stream)
{
    if (!c) return QRM_E_INVALID;
    if (!o) return fail(c, QRM_E_INVALID, "opt is NULL");
    if (o->device != c->device) return fail(c, QRM_E_INVALID, "the plan belongs to another device");
    if (!d_scale || !aligned_to(d_scale, 4)) return fail(c, QRM_E_INVALID, "d_scale is NULL or not aligned to its elements");
    qrm_status st = check_grads(c, o, h_grads);
    if (st != QRM_OK) return st;
    const int n = (int)o->first_piece.size() - 1;
    if (n <= 0) return QRM_OK;
    if (!h_outs) return fail(c, QRM_E_INVALID, "h_outs is NULL");
    for (int i = 0; i < n; ++i) {
        if (!h_grads[i] != !h_outs[i]) return fail(c, QRM_E_INVALID, "a gradient without an output, or the reverse");
        if (!aligned_to(h_outs[i], type_bytes(o->types.grad))) return fail(c, QRM_E_INVALID, "a pointer is not aligned to its elements");
    }
    if ((st = check_outs(c, o, h_outs)) != QRM_OK || (st = start(c)) != QRM_OK) return st;
    for (int i = 0; i < n; i += kScaleGrads) {
        const int count = std::min(n - i, kScaleGrads);
        const uint32_t from = o->first_piece[i], to = o->first_piece[i + count];
        if (from == to) continue;
        hipError_t e = launch_scale_grads(o->types.grad, o->tensors, o->pieces, from, to - from, i, h_grads + i, h_outs + i, count, d_scale, (hipStream_t)stream);
        if (e != hipSuccess) {
            char what[64];
            snprintf(what, sizeof what, "scale_grads launch of tensor %d and those behind it", i);
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

qrm_status qrm_attention(qrm_ctx *c, const qrm_attention_desc *desc, const void *d_q, const void *d_k, const void *d_v, const int32_t *d_q_len, const int32_t *d_k_len,
                         void *d_o, float *d_lse, void *stream)
{
    if (!c) return QRM_E_INVALID;
    AttnCheck a;
    qrm_status st = check_attention(c, desc, &a);
    if (st != QRM_OK) return st;
    const qrm_attention_desc &d = a.d;
    if (d.N == 0 || d.Lq == 0) return QRM_OK;
    if (!d_q || !d_o || (d.Lk && (!d_k || !d_v))) return fail(c, QRM_E_INVALID, "d_q / d_k / d_v / d_o is NULL");
    if (d_o == d_q || d_o == d_k || d_o == d_v) return fail(c, QRM_E_INVALID, "d_o is an input");
    const int size = type_bytes(d.type);
    if (common_alignment({d_q, d_k, d_v, d_o}) < size || !aligned_to(d_lse, 4) || !aligned_to(d_q_len, 4) || !aligned_to(d_k_len, 4))
        return fail(c, QRM_E_INVALID, "a pointer is not aligned to its elements");
    const AttnCut cut = plan_attention(d, a.wide, c->num_cu);
    if (std::max(cut.threads(d), cut.join_threads(d)) >= kLaunchThreads) return fail(c, QRM_E_UNSUPPORTED, kTooManyRows);
    Workspace w;
    const AttnTensor q = place(a, a.q, d.Lq, d.heads, {d_q}, 1, &w), k = place(a, a.k, d.Lk, d.kv_heads, {d_k}, 1, &w), v = place(a, a.v, d.Lk, d.kv_heads, {d_v}, 1, &w),
                     o = place(a, a.o, d.Lq, d.heads, {d_o}, 1, &w);
    const size_t part = w.take(cut.part_bytes(d)), sums = w.take(cut.sums_bytes(d));
    if ((st = start(c)) != QRM_OK) return st;
    QrmSlot *slot = nullptr;
    const hipStream_t s = (hipStream_t)stream;
    if (w.bytes && (st = get_slot(c, s, w.bytes, &slot)) != QRM_OK) return st;
    uint8_t *const ws = slot ? (uint8_t *)slot->ws : nullptr;
    AttnArgs g = attention_args(a, q, k, v, o, d_q_len, d_k_len);
    cut_to(&g, cut);
    g.lse = d_lse;
    g.part = (float *)(ws + part), g.part_sums = (float *)(ws + sums);
    hipError_t e = hipSuccess;
    auto in = [&](const AttnTensor &t, const AttnRows &r, const void *p, int64_t L, int heads) -> const void * {
        if (!t.copied) return p;
        if (e == hipSuccess && L) e = launch_attention_copy(d.type, false, r, const_cast<void *>(p), ws + t.at, d.N, L, heads, d.D, a.wide, s);
        return ws + t.at;
    };
    g.q = in(q, a.q, d_q, d.Lq, d.heads);
    g.k = in(k, a.k, d_k, d.Lk, d.kv_heads);
    g.v = in(v, a.v, d_v, d.Lk, d.kv_heads);
    g.o = o.copied ? ws + o.at : d_o;
    if (e == hipSuccess) e = launch_attention(d.type, cut.kind, g, s);
    if (e == hipSuccess && cut.splits > 1) e = launch_attention_join(d.type, g, cut, s);
    if (e == hipSuccess && o.copied) e = launch_attention_copy(d.type, true, a.o, d_o, g.o, d.N, d.Lq, d.heads, d.D, a.wide, s);
    if (slot) st = slot_done(c, slot, s, true);
    return e == hipSuccess ? st : hip_fail(c, e, "attention launch");
}

qrm_status qrm_attention_backward(qrm_ctx *c, const qrm_attention_desc *desc, const void *d_q, const void *d_k, const void *d_v, const void *d_o, const void *d_do,
                                  const float *d_lse, const int32_t *d_q_len, const int32_t *d_k_len, void *d_dq, void *d_dk, void *d_dv, void *stream)
{
    if (!c) return QRM_E_INVALID;
    AttnCheck a;
    qrm_status st = check_attention(c, desc, &a);
    if (st != QRM_OK) return st;
    const qrm_attention_desc &d = a.d;
    if (!d_dq && !d_dk && !d_dv) return fail(c, QRM_E_INVALID, "no output is asked for");
    if (d.Lq == 0) d_dq = nullptr;
    if (d.Lk == 0) d_dk = d_dv = nullptr;
    if (d.N == 0 || (!d_dq && !d_dk && !d_dv)) return QRM_OK;
    if ((d.Lq && (!d_q || !d_o || !d_do || !d_lse)) || (d.Lk && (!d_k || !d_v))) return fail(c, QRM_E_INVALID, "d_q / d_k / d_v / d_o / d_do / d_lse is NULL");
    const void *const inputs[] = {d_q, d_k, d_v, d_o, d_do}, *const outputs[] = {d_dq, d_dk, d_dv};
    for (int i = 0; i < 3; ++i) {
        for (const void *p : inputs)
            if (outputs[i] && outputs[i] == p) return fail(c, QRM_E_INVALID, "an output is an input");
        if (outputs[i] && outputs[i] == outputs[(i + 1) % 3]) return fail(c, QRM_E_INVALID, "two outputs are one");
    }
    const int size = type_bytes(d.type);
    if (common_alignment({d_q, d_k, d_v, d_o, d_do, d_dq, d_dk, d_dv}) < size || !aligned_to(d_lse, 4) || !aligned_to(d_q_len, 4) || !aligned_to(d_k_len, 4))
        return fail(c, QRM_E_INVALID, "a pointer is not aligned to its elements");
    AttnCut by_q{}, by_k{};
    plan_attention_backward(d, a.wide, c->num_cu, &by_q, &by_k);
    if (std::max(by_q.threads(d) + by_k.threads(d), by_q.join_threads(d) + 2 * by_k.join_threads(d)) >= kLaunchThreads) return fail(c, QRM_E_UNSUPPORTED, kTooManyRows);
    Workspace w;
    const size_t q_rows = (size_t)d.N * d.heads * d.Lq, k_rows = (size_t)d.N * d.kv_heads * d.Lk;
    // (a copied tensor's gradient is written behind its copy)
    const AttnTensor q = place(a, a.q, d.Lq, d.heads, {d_q, d_dq}, 2, &w), k = place(a, a.k, d.Lk, d.kv_heads, {d_k, d_dk}, 2, &w),
                     v = place(a, a.v, d.Lk, d.kv_heads, {d_v, d_dv}, 2, &w), y = place(a, a.o, d.Lq, d.heads, {d_do}, 1, &w);
    const size_t row_lse = w.take(q_rows * 4), row_delta = w.take(q_rows * 4);
    const size_t part_q = w.take(d_dq ? by_q.part_bytes(d) : 0), part_k = w.take(d_dk ? by_k.part_bytes(d) : 0), part_v = w.take(d_dv ? by_k.part_bytes(d) : 0);
    if ((st = start(c)) != QRM_OK) return st;
    QrmSlot *slot = nullptr;
    const hipStream_t s = (hipStream_t)stream;
    if ((st = get_slot(c, s, w.bytes, &slot)) != QRM_OK) return st;
    uint8_t *const ws = (uint8_t *)slot->ws;
    AttnArgs g = attention_args(a, q, k, v, y, d_q_len, d_k_len);
    hipError_t e = hipSuccess;
    auto in = [&](const AttnTensor &t, const AttnRows &r, const void *p, int64_t L, int heads) -> const void * {
        if (!t.copied) return p;
        if (e == hipSuccess && L) e = launch_attention_copy(d.type, false, r, const_cast<void *>(p), ws + t.at, d.N, L, heads, d.D, a.wide, s);
        return ws + t.at;
    };
    auto out = [&](const AttnTensor &t, void *p, size_t rows) -> void * { return !p ? nullptr : t.copied ? ws + t.at + rows * a.wide * size : p; };
    auto back = [&](const AttnTensor &t, const AttnRows &r, void *p, void *from, int64_t L, int heads) {
        if (e == hipSuccess && p && t.copied) e = launch_attention_copy(d.type, true, r, p, from, d.N, L, heads, d.D, a.wide, s);
    };
    g.q = in(q, a.q, d_q, d.Lq, d.heads);
    g.k = in(k, a.k, d_k, d.Lk, d.kv_heads);
    g.v = in(v, a.v, d_v, d.Lk, d.kv_heads);
    g.dy = in(y, a.o, d_do, d.Lq, d.heads);
    g.dq = out(q, d_dq, q_rows), g.dk = out(k, d_dk, k_rows), g.dv = out(v, d_dv, k_rows);
    g.row_lse = (float *)(ws + row_lse), g.row_delta = (float *)(ws + row_delta);
    g.part = (float *)(ws + part_q), g.part_k = (float *)(ws + part_k), g.part_v = (float *)(ws + part_v);
    if (e == hipSuccess && d.Lq) e = launch_attention_rows(d, d_o, d_do, d_lse, d_q_len, (float *)(ws + row_lse), (float *)(ws + row_delta), s);
    AttnArgs gq = g, gk = g;
    cut_to(&gq, by_q);
    cut_to(&gk, by_k);
    if (e == hipSuccess) e = launch_attention_backward(d.type, gq, gk, s);
    if (e == hipSuccess) e = launch_attention_add(d.type, gq, by_q, gk, by_k, s);
    back(q, a.q, d_dq, g.dq, d.Lq, d.heads);
    back(k, a.k, d_dk, g.dk, d.Lk, d.kv_heads);
    back(v, a.v, d_dv, g.dv, d.Lk, d.kv_heads);
    st = slot_done(c, slot, s, true);
    return e == hipSuccess ? st : hip_fail(c, e, "attention_backward launch");
}

} // extern "C"
