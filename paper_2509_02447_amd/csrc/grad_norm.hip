// The norm of all gradients of a step with the factor that clips it (qrm_adamw_grad_norm), and gradients times a factor (qrm_adamw_scale_grads).
//
// A wavefront takes pieces of 4096 elements from the optimiser's table; squares and sums are taken in 64 bits, as wide as no square of a gradient
// overflows.  One launch: the workgroup that is done last adds the others' sums up, in their order.  Bound by memory: a gradient is read once, a
// piece a wavefront (16 KB of f32, 8 KB of 16 bits) under way before the first is used (50 M elements of bf16, 100 MB: 28 us, 3.5 TB/s; 60 thousand of f32 in one workgroup: 5.7 us); the factor is
// applied in 32 us (200 MB, 6.2 TB/s).
#include "qrm_train.h"

#include <algorithm>

namespace qrm {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kScaleThreads = 256;
constexpr int kSet = 16, kLine = 32; // workgroups that share a count; words from one count to the next

template <int COUNT> struct Grads {
    const void *p[COUNT];
};
template <int COUNT> struct GradsOut {
    const void *p[COUNT];
    void *out[COUNT];
};

__device__ __forceinline__ double wave_sum(double v)
{
    for (int apart = 32; apart; apart /= 2) v += __shfl_xor(v, apart);
    return v;
}

template <typename T, int COUNT>
__global__ __launch_bounds__(kThreads) void grad_norm_kernel(const AdamwTensor *tensors, const uint2 *pieces, uint32_t count, uint32_t t0, Grads<COUNT> grads, NormParts parts)
{
    __shared__ double sums[kWaves];
    __shared__ bool last;
    constexpr int V = 16 / (int)sizeof(T), TIMES = kAdamwPiece / (64 * V);
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    double sum = 0.0;
    for (uint32_t i = wave * gridDim.x + blockIdx.x; i < count; i += gridDim.x * kWaves) {
        const uint2 piece = pieces[i];
        const T *const grad = (const T *)grads.p[piece.x - t0];
        if (!grad) continue;
        const int64_t first = (int64_t)piece.y * kAdamwPiece;
        const int n = (int)min((int64_t)kAdamwPiece, tensors[piece.x].n - first);
        const T *const p = grad + first;
        int done = 0;
        if (((uintptr_t)p & 15) == 0) {
            done = n / V * V;
            Pack<T, V> e[TIMES];
            if (n == kAdamwPiece) { // all on their way before the first is used
#pragma unroll
                for (int k = 0; k < TIMES; ++k) e[k] = load_pack<T, V>(p + (k * 64 + lane) * V);
            } else {
#pragma unroll
                for (int k = 0; k < TIMES; ++k) e[k] = (k * 64 + lane) * V < done ? load_pack<T, V>(p + (k * 64 + lane) * V) : Pack<T, V>{};
            }
            double some[2] = {};
#pragma unroll
            for (int k = 0; k < TIMES; ++k)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const double g = (double)(float)e[k].e[v];
                    some[v & 1] = fma(g, g, some[v & 1]);
                }
            sum += some[0] + some[1];
        }
        for (int k = done + lane; k < n; k += 64) {
            const double g = (double)(float)p[k];
            sum = fma(g, g, sum);
        }
    }
    sum = wave_sum(sum);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = 0.0;
    if (threadIdx.x == 0) {
        for (int w = 0; w < kWaves; ++w) sum += sums[w];
        last = gridDim.x == 1 && parts.total == 1;
        if (!last) {
            // stored past the L2s; a sum has arrived before its workgroup is counted, and those of earlier launches are there
            __hip_atomic_store(parts.sums + parts.first + blockIdx.x, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if (parts.ends) {
                // (additions to one word follow each other: sixteen workgroups share one, in a line of its own, and the last of them counts on in the first word)
                const auto counted = [](uint32_t *word, uint32_t all) {
                    const bool full = __hip_atomic_fetch_add(word, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == all;
                    if (full) __hip_atomic_store(word, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    return full;
                };
                const uint32_t sets = (gridDim.x + kSet - 1) / kSet, set = blockIdx.x % sets;
                last = counted(parts.done + (1 + set) * kLine, gridDim.x / sets + (set < gridDim.x % sets)) && counted(parts.done, sets);
            }
        }
    }
    __syncthreads();
    if (!last) return;
    if (parts.total > 1) {
        sum = 0.0;
        for (uint32_t i = threadIdx.x; i < parts.total; i += kThreads) sum += __hip_atomic_load(parts.sums + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        sum = wave_sum(sum);
        if (lane == 0) sums[wave] = sum;
        __syncthreads();
        sum = 0.0;
        if (threadIdx.x == 0)
            for (int w = 0; w < kWaves; ++w) sum += sums[w];
    }
    if (threadIdx.x) return;
    const double u = parts.unscale ? (double)*parts.unscale : 1.0, norm = sqrt(sum) * u, part = parts.max_norm / norm;
    if (parts.norm) *parts.norm = (float)norm;
    if (parts.scale) *parts.scale = (float)(part >= 1.0 ? u : u * part); // (a norm that is not a number: neither is the factor)
}

template <typename T, int COUNT>
__global__ __launch_bounds__(kScaleThreads) void scale_grads_kernel(const AdamwTensor *tensors, const uint2 *pieces, uint32_t t0, GradsOut<COUNT> grads, const float *scale)
{
    constexpr int V = 16 / (int)sizeof(T), TIMES = kAdamwPiece / (kScaleThreads * V);
    const uint2 piece = pieces[blockIdx.x];
    const T *grad = (const T *)grads.p[piece.x - t0];
    if (!grad) return;
    T *out = (T *)grads.out[piece.x - t0];
    const float by = *scale;
    if (by == 1.f && out == grad) return;
    const int64_t first = (int64_t)piece.y * kAdamwPiece;
    const int n = (int)min((int64_t)kAdamwPiece, tensors[piece.x].n - first);
    grad += first;
    out += first;
    int done = 0;
    if ((((uintptr_t)grad | (uintptr_t)out) & 15) == 0) {
        done = n / V * V;
        Pack<T, V> e[TIMES];
#pragma unroll
        for (int k = 0; k < TIMES; ++k) {
            const int i = (k * kScaleThreads + threadIdx.x) * V;
            if (i < done) e[k] = load_pack<T, V>(grad + i);
        }
#pragma unroll
        for (int k = 0; k < TIMES; ++k) {
            const int i = (k * kScaleThreads + threadIdx.x) * V;
#pragma unroll
            for (int v = 0; v < V; ++v) e[k].e[v] = (T)((float)e[k].e[v] * by);
            if (i < done) store_pack<T, V>(out + i, e[k]);
        }
    }
    for (int i = done + threadIdx.x; i < n; i += kScaleThreads) out[i] = (T)((float)grad[i] * by);
}

template <int COUNT>
hipError_t norm_counted(int type, const AdamwTensor *tensors, const uint2 *pieces, uint32_t count, uint32_t t0, const void *const *grads, int n_grads, const NormParts &parts, uint32_t blocks,
                        hipStream_t s)
{
    Grads<COUNT> g;
    for (int i = 0; i < COUNT; ++i) g.p[i] = i < n_grads ? grads[i] : nullptr;
    return with_type(type, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        hipLaunchKernelGGL((grad_norm_kernel<T, COUNT>), dim3(blocks), dim3(kThreads), 0, s, tensors, pieces, count, t0, g, parts);
        return hipGetLastError();
    });
}

template <int COUNT>
hipError_t scale_counted(int type, const AdamwTensor *tensors, const uint2 *pieces, uint32_t count, uint32_t t0, const void *const *grads, void *const *outs, int n_grads, const float *scale,
                         hipStream_t s)
{
    GradsOut<COUNT> g;
    for (int i = 0; i < COUNT; ++i) g.p[i] = i < n_grads ? grads[i] : nullptr, g.out[i] = i < n_grads ? outs[i] : nullptr;
    return with_type(type, [&](auto *p) {
        using T = std::remove_pointer_t<decltype(p)>;
        hipLaunchKernelGGL((scale_grads_kernel<T, COUNT>), dim3(count), dim3(kScaleThreads), 0, s, tensors, pieces, t0, g, scale);
        return hipGetLastError();
    });
}

} // namespace

// A workgroup to a compute unit at most (the counts of a workspace serve 16 times 31), one where its wavefronts have few pieces.
uint32_t norm_blocks(uint32_t pieces) { return pieces <= 4 * kWaves ? 1 : std::min<uint32_t>((pieces + kWaves - 1) / kWaves, 256); }

hipError_t launch_grad_norm(int type, const AdamwTensor *tensors, const uint2 *pieces, uint32_t first, uint32_t count, uint32_t t0, const void *const *grads, int n_grads,
                            const NormParts &parts, hipStream_t s)
{
    return n_grads <= 32 ? norm_counted<32>(type, tensors, pieces + first, count, t0, grads, n_grads, parts, norm_blocks(count), s)
                         : norm_counted<kAdamwGrads>(type, tensors, pieces + first, count, t0, grads, n_grads, parts, norm_blocks(count), s);
}

hipError_t launch_scale_grads(int type, const AdamwTensor *tensors, const uint2 *pieces, uint32_t first, uint32_t count, uint32_t t0, const void *const *grads, void *const *outs, int n_grads,
                              const float *scale, hipStream_t s)
{
    return n_grads <= 32 ? scale_counted<32>(type, tensors, pieces + first, count, t0, grads, outs, n_grads, scale, s)
                         : scale_counted<kScaleGrads>(type, tensors, pieces + first, count, t0, grads, outs, n_grads, scale, s);
}

} // namespace qrm
