// One AdamW step over many tensors (qrm_adamw_step) and the values of 8-bit moments (qrm_unpack_moment).
//
// A workgroup takes a piece of 4096 elements of one tensor; which one, a table of the plan says, so that one launch does hundreds of tensors of
// any sizes.  Every element is read and written once; nothing is shared between elements but a block's scale of 8-bit moments, which is the largest of 256
// neighbours: four to a lane, one block to a wavefront, no shared memory.  All of a thread's loads are on their way before the first is used.  Bound by memory: 28
// bytes an element in 32 bits (200 million 1026 us, 5.5 TB/s; a large copy passes 5.1), 16 with 8-bit moments beside 16-bit gradients and a 16-bit copy (50
// million 143 us, 5.6 TB/s).  60 thousand elements take 5.1 us: three dependent loads (piece, tensor, data) and the launch.
#include "qrm_train.h"

#include <type_traits>

namespace qrm {
namespace {

constexpr int kThreads = 256;

template <int COUNT> struct Grads {
    const void *p[COUNT];
};

struct Rates { // of a tensor, in a step
    float beta1, rest1, beta2, rest2, eps, keep, rate, root, scale;
};

__device__ __forceinline__ Rates rates_of(const AdamwStep &s, const AdamwTensor &t)
{
    return Rates{s.beta1, s.rest1, s.beta2, s.rest2, s.eps, 1.f - s.lr * t.lr_scale * t.weight_decay, s.rate * t.lr_scale, s.root, s.grad_scale ? *s.grad_scale : 1.f};
}

__device__ __forceinline__ void moments(const Rates &r, float g, float &m, float &v)
{
    g *= r.scale;
    m = m * r.beta1 + g * r.rest1;
    v = v * r.beta2 + g * g * r.rest2;
}

template <int V, bool STREAM = false> __device__ __forceinline__ void store_copy(void *copy, int type, int64_t i, const float (&p)[V])
{
    if (type == QRM_BF16) {
        Pack<bf16_t, V> c;
#pragma unroll
        for (int k = 0; k < V; ++k) c.e[k] = (bf16_t)p[k];
        store_pack<bf16_t, V, STREAM>((bf16_t *)copy + i, c);
    } else {
        Pack<f16_t, V> c;
#pragma unroll
        for (int k = 0; k < V; ++k) c.e[k] = (f16_t)p[k];
        store_pack<f16_t, V, STREAM>((f16_t *)copy + i, c);
    }
}

// What a thread holds of a piece: V neighbouring elements.
template <typename TP, typename TG, int V> struct Some {
    Pack<TP, V> p;
    Pack<TG, V> g;
    Pack<float, V> m, v;
};
template <typename TP, typename TG, int V, bool STREAM> __device__ __forceinline__ Some<TP, TG, V> load_some(const AdamwTensor &t, const TG *grad, int64_t i)
{
    return Some<TP, TG, V>{load_pack<TP, V, STREAM>((const TP *)t.p + i), load_pack<TG, V, STREAM>(grad + i), load_pack<float, V, STREAM>((const float *)t.m + i),
                           load_pack<float, V, STREAM>((const float *)t.v + i)};
}
template <typename TP, typename TG, int V, bool STREAM> __device__ __forceinline__ void step_some(const AdamwTensor &t, const Rates &r, int copy_type, int64_t i, Some<TP, TG, V> e)
{
    float w[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        moments(r, (float)e.g.e[k], e.m.e[k], e.v.e[k]);
        w[k] = (float)e.p.e[k] * r.keep - r.rate * (e.m.e[k] / (sqrtf(e.v.e[k]) * r.root + r.eps));
        e.p.e[k] = (TP)w[k];
    }
    store_pack<TP, V, STREAM>((TP *)t.p + i, e.p);
    store_pack<float, V, STREAM>((float *)t.m + i, e.m);
    store_pack<float, V, STREAM>((float *)t.v + i, e.v);
    if (t.copy) store_copy<V, STREAM>(t.copy, copy_type, i, w);
}

__device__ __forceinline__ bool aligned(const void *p, int bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// A multiple of four elements of every array lies on a boundary that one load or store needs.
template <typename TP, typename TG, typename TM> __device__ __forceinline__ bool wide_ok(const AdamwTensor &t, const TG *grad)
{
    return aligned(t.p, 4 * sizeof(TP)) && aligned(grad, 4 * sizeof(TG)) && aligned(t.m, 4 * sizeof(TM)) && aligned(t.v, 4 * sizeof(TM)) &&
           aligned(t.copy, 8);
}

template <typename TP, typename TG, int COUNT, bool STREAM>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const AdamwTensor *tensors, const uint2 *pieces, uint32_t t0, Grads<COUNT> grads, AdamwStep s, int copy_type)
{
    const uint2 piece = pieces[blockIdx.x];
    const AdamwTensor t = tensors[piece.x];
    const TG *grad = (const TG *)grads.p[piece.x - t0];
    if (!grad) return;
    const Rates r = rates_of(s, t);
    const int64_t first = (int64_t)piece.y * kAdamwPiece, last = min(first + kAdamwPiece, t.n);
    constexpr int kTimes = kAdamwPiece / (kThreads * 4);
    if (!wide_ok<TP, TG, float>(t, grad)) {
        for (int64_t i = first + threadIdx.x; i < last; i += kThreads) step_some<TP, TG, 1, false>(t, r, copy_type, i, load_some<TP, TG, 1, false>(t, grad, i));
        return;
    }
    // all on their way before the first is used; what is behind the end is the last four elements' that are there
    const int64_t quads = first + (last - first) / 4 * 4;
    if (quads > first) {
        Some<TP, TG, 4> e[kTimes];
#pragma unroll
        for (int j = 0; j < kTimes; ++j) e[j] = load_some<TP, TG, 4, STREAM>(t, grad, min(first + (j * kThreads + threadIdx.x) * 4, quads - 4));
#pragma unroll
        for (int j = 0; j < kTimes; ++j) {
            const int64_t i = first + (j * kThreads + threadIdx.x) * 4;
            if (i < quads) step_some<TP, TG, 4, STREAM>(t, r, copy_type, i, e[j]);
        }
    }
    if (quads + threadIdx.x < last) step_some<TP, TG, 1, false>(t, r, copy_type, quads + threadIdx.x, load_some<TP, TG, 1, false>(t, grad, quads + threadIdx.x));
}

// ---------------------------------------------------------------- moments in 8 bits

// Codes as numbers, before the block's scale.
__device__ __forceinline__ float square_m(int8_t c) { return (float)c * fabsf((float)c); }
__device__ __forceinline__ float square_u(uint8_t c) { return (float)c * (float)c; }
constexpr float kStepM = 1.f / 16129.f, kStepU = 1.f / 65025.f; // 1 / 127^2, 1 / 255^2

// The larger of v and another lane's, of numbers >= 0 by their bits: a NaN counts as larger than all.
template <int CTRL> __device__ __forceinline__ int max_lane(int v) { return max(v, __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true)); }
__device__ __forceinline__ float wave_max(int v)
{
    v = max_lane<0xB1>(v);  // pairs, fours, halves of a row of 16, rows
    v = max_lane<0x4E>(v);
    v = max_lane<0x141>(v);
    v = max_lane<0x140>(v);
    v = max(v, __shfl_xor(v, 16));
    return __int_as_float(max(v, __shfl_xor(v, 32)));
}
__device__ __forceinline__ int magnitude(float v) { return __float_as_int(v) & 0x7fffffff; }

// What a lane holds of a block: four neighbouring elements.
template <typename TP, typename TG> struct Quad {
    Pack<TP, 4> p;
    Pack<TG, 4> g;
    Pack<int8_t, 4> m;
    Pack<uint8_t, 4> u;
    float scale_m, scale_u;
};

// One step of a wavefront's block; the scales come back the same in all lanes, w the parameters in 32 bits.  The arithmetic takes the hardware's roots and
// inverses as they are (1 ulp): rounded exactly, they would take longer than the memory does.  They know no numbers below 2^-126: blocks with such a v take
// the library's root, moments of a tiny scale are lifted first.
template <typename TP, typename TG> __device__ __forceinline__ void step_block(const Rates &r, Quad<TP, TG> &q, float (&w)[4])
{
    const float sm = q.scale_m * kStepM, su = q.scale_u * kStepU;
    float m[4], v[4], u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        m[k] = square_m(q.m.e[k]) * sm;
        const float root = square_u(q.u.e[k]) * su;
        v[k] = root * root;
        moments(r, (float)q.g.e[k], m[k], v[k]);
        u[k] = __builtin_amdgcn_sqrtf(v[k]);
    }
    if (__any(fminf(fminf(v[0], v[1]), fminf(v[2], v[3])) < 0x1p-100f)) {
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = sqrtf(v[k]);
    }
    int top_m = 0, top_u = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        w[k] = (float)q.p.e[k] * r.keep - r.rate * (m[k] * __builtin_amdgcn_rcpf(u[k] * r.root + r.eps));
        q.p.e[k] = (TP)w[k];
        top_m = max(top_m, magnitude(m[k]));
        top_u = max(top_u, magnitude(u[k]));
    }
    q.scale_m = wave_max(top_m);
    q.scale_u = wave_max(top_u);
    float of_m = q.scale_m;
    if (of_m < 0x1p-100f) {
        of_m *= 0x1p100f;
#pragma unroll
        for (int k = 0; k < 4; ++k) m[k] *= 0x1p100f;
    }
    const float inv_m = of_m > 0.f ? 16129.f * __builtin_amdgcn_rcpf(of_m) : 0.f, inv_u = q.scale_u > 0.f ? 65025.f * __builtin_amdgcn_rcpf(q.scale_u) : 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        q.m.e[k] = (int8_t)(int)copysignf(rintf(__builtin_amdgcn_sqrtf(fabsf(m[k]) * inv_m)), m[k]);
        const float y = rintf(__builtin_amdgcn_sqrtf(u[k] * inv_u));
        q.u.e[k] = (uint8_t)(int)(u[k] > 0.f ? fmaxf(y, 1.f) : 0.f);
    }
}

template <typename TP, typename TG, int COUNT, bool STREAM>
__global__ __launch_bounds__(kThreads) void adamw8_kernel(const AdamwTensor *tensors, const uint2 *pieces, uint32_t t0, Grads<COUNT> grads, AdamwStep s, int copy_type)
{
    constexpr int kBlocks = kAdamwPiece / (kThreads / 64) / QRM_MOMENT_BLOCK; // of a wavefront, side by side
    const uint2 piece = pieces[blockIdx.x];
    const AdamwTensor t = tensors[piece.x];
    const TG *grad = (const TG *)grads.p[piece.x - t0];
    if (!grad) return;
    const Rates r = rates_of(s, t);
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const int64_t first = (int64_t)piece.y * kAdamwPiece + wave * (kBlocks * QRM_MOMENT_BLOCK), last = min((int64_t)(piece.y + 1) * kAdamwPiece, t.n);
    float *const scales_m = t.m_scale + first / QRM_MOMENT_BLOCK, *const scales_u = t.v_scale + first / QRM_MOMENT_BLOCK;
    TP *const p = (TP *)t.p + first;
    const TG *const g = grad + first;
    int8_t *const m = (int8_t *)t.m + first;
    uint8_t *const u = (uint8_t *)t.v + first;
    if (first + kBlocks * QRM_MOMENT_BLOCK <= last && wide_ok<TP, TG, uint8_t>(t, grad)) {
        Quad<TP, TG> q[kBlocks]; // all on their way before the first is used
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            const int i = b * QRM_MOMENT_BLOCK + lane * 4;
            q[b].scale_m = scales_m[b];
            q[b].scale_u = scales_u[b];
            q[b].p = load_pack<TP, 4, STREAM>(p + i);
            q[b].g = load_pack<TG, 4, STREAM>(g + i);
            q[b].m = load_pack<int8_t, 4>(m + i);
            q[b].u = load_pack<uint8_t, 4>(u + i);
        }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            const int i = b * QRM_MOMENT_BLOCK + lane * 4;
            float w[4];
            step_block<TP, TG>(r, q[b], w);
            store_pack<TP, 4, STREAM>(p + i, q[b].p);
            store_pack<int8_t, 4>(m + i, q[b].m);
            store_pack<uint8_t, 4>(u + i, q[b].u);
            if (t.copy) store_copy<4, STREAM>(t.copy, copy_type, first + i, w);
            if (lane == 0) scales_m[b] = q[b].scale_m, scales_u[b] = q[b].scale_u;
        }
        return;
    }
    for (int b = 0; b < kBlocks && first + b * QRM_MOMENT_BLOCK < last; ++b) {
        const int i = b * QRM_MOMENT_BLOCK + lane * 4, here = (int)max((int64_t)0, min((int64_t)4, last - first - i));
        Quad<TP, TG> q{}; // (elements that are not there: zeros, of no weight in the largest)
        q.scale_m = scales_m[b];
        q.scale_u = scales_u[b];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < here) q.p.e[k] = p[i + k], q.g.e[k] = g[i + k], q.m.e[k] = m[i + k], q.u.e[k] = u[i + k];
        float w[4];
        step_block<TP, TG>(r, q, w);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < here) {
                p[i + k] = q.p.e[k], m[i + k] = q.m.e[k], u[i + k] = q.u.e[k];
                const float one[1] = {w[k]};
                if (t.copy) store_copy<1>(t.copy, copy_type, first + i + k, one);
            }
        if (lane == 0) scales_m[b] = q.scale_m, scales_u[b] = q.scale_u;
    }
}

// Sixteen codes a thread, 4096 a workgroup.  50 million to bf16: 28 us, 5.3 TB/s.
constexpr int kUnpack = 16;
template <typename T> __global__ __launch_bounds__(kThreads) void unpack_moment_kernel(int moment, const uint8_t *codes, const float *scales, int64_t n, T *out)
{
    const int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kUnpack;
    if (i >= n) return;
    const float scale = scales[i / QRM_MOMENT_BLOCK] * (moment ? kStepU : kStepM);
    auto value = [&](uint8_t c) {
        if (moment == 0) return (T)(square_m((int8_t)c) * scale);
        const float u = square_u(c) * scale;
        return (T)(u * u);
    };
    if (i + kUnpack <= n && aligned(codes, kUnpack) && aligned(out, 16)) {
        constexpr int V = 16 / sizeof(T);
        const Pack<uint8_t, kUnpack> c = load_pack<uint8_t, kUnpack>(codes + i);
#pragma unroll
        for (int j = 0; j < kUnpack; j += V) {
            Pack<T, V> v;
#pragma unroll
            for (int k = 0; k < V; ++k) v.e[k] = value(c.e[j + k]);
            store_pack<T, V>(out + i + j, v);
        }
    } else {
        for (int k = 0; k < kUnpack && i + k < n; ++k) out[i + k] = value(codes[i + k]);
    }
}

template <int COUNT>
hipError_t launch_counted(const AdamwTypes &t, const AdamwTensor *tensors, const uint2 *pieces, uint32_t count, uint32_t t0, const void *const *grads, int n_grads,
                          const AdamwStep &step, hipStream_t s)
{
    Grads<COUNT> g;
    for (int i = 0; i < COUNT; ++i) g.p[i] = i < n_grads ? grads[i] : nullptr;
    return with_type(t.param, [&](auto *np) {
        return with_type(t.grad, [&](auto *ng) {
            using TP = std::remove_pointer_t<decltype(np)>;
            using TG = std::remove_pointer_t<decltype(ng)>;
            auto launch = [&](auto stream) {
                constexpr bool STREAM = decltype(stream)::value;
                if (t.bits == 32)
                    hipLaunchKernelGGL((adamw_kernel<TP, TG, COUNT, STREAM>), dim3(count), dim3(kThreads), 0, s, tensors, pieces, t0, g, step, t.copy);
                else
                    hipLaunchKernelGGL((adamw8_kernel<TP, TG, COUNT, STREAM>), dim3(count), dim3(kThreads), 0, s, tensors, pieces, t0, g, step, t.copy);
            };
            t.stream ? launch(std::true_type()) : launch(std::false_type());
            return hipGetLastError();
        });
    });
}

} // namespace

hipError_t launch_adamw(const AdamwTypes &t, const AdamwTensor *tensors, const uint2 *pieces, uint32_t first, uint32_t count, uint32_t t0,
                        const void *const *grads, int n_grads, const AdamwStep &step, hipStream_t s)
{
    // (arguments are copied at every launch: short lists take short ones)
    return n_grads <= 32 ? launch_counted<32>(t, tensors, pieces + first, count, t0, grads, n_grads, step, s)
                         : launch_counted<kAdamwGrads>(t, tensors, pieces + first, count, t0, grads, n_grads, step, s);
}

hipError_t launch_unpack_moment(int moment, const void *codes, const float *scales, int64_t n, int out_type, void *out, hipStream_t s)
{
    const dim3 grid((uint32_t)((n + kUnpack * kThreads - 1) / (kUnpack * kThreads)));
    if (out_type == QRM_F32)
        hipLaunchKernelGGL(unpack_moment_kernel<float>, grid, dim3(kThreads), 0, s, moment, (const uint8_t *)codes, scales, n, (float *)out);
    else
        hipLaunchKernelGGL(unpack_moment_kernel<bf16_t>, grid, dim3(kThreads), 0, s, moment, (const uint8_t *)codes, scales, n, (bf16_t *)out);
    return hipGetLastError();
}

} // namespace qrm
