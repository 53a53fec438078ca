// Message loss with its gradient (qrm_message_loss).
//
// A lane takes a symbol, 2^k lanes an image: the image's expected number of wrong symbols, which every bit's gradient depends on, is a sum over
// neighbouring lanes.  Bound by launch latency up to thousands of images, by memory beyond (9 bytes a bit).
#include "qrm_train.h"

#include <algorithm>
#include <type_traits>

namespace qrm {
namespace {

constexpr int kThreads = 256, kSmallThreads = 1024;

struct LossArgs {
    const float *logits;
    const uint8_t *target;
    int64_t target_stride, N;
    int n_bits, n, t, lanes; // lanes: of an image, a power of two
    float weight, per_bit, per_image; // 1 / (N n_bits), weight / N
    float *loss, *grad;
    int32_t *bit_errors, *symbol_errors;
    double *partial; // [workgroups], or null: one workgroup, which writes the loss
};

template <int M> struct Symbol {
    float x[M];        // logits, turned so that the right side is above zero
    uint32_t ones;     // target bits
    int wrong;         // hard bits that differ
    float bce, right;  // sum of -log sigmoid(x); chance that all bits are right
};

template <int M> __device__ __forceinline__ Symbol<M> read_symbol(const LossArgs &a, int64_t image, int j)
{
    Symbol<M> s;
    const float *z = a.logits + image * a.n_bits + j * M;
    const uint8_t *target = a.target + image * a.target_stride + j * M;
    s.ones = 0;
    s.wrong = 0;
    s.bce = 0.f;
#pragma unroll
    for (int b = 0; b < M; ++b) {
        const bool one = target[b] != 0;
        const float v = z[b];
        s.ones |= (uint32_t)one << b;
        s.wrong += (v > 0.f) != one;
        s.x[b] = one ? v : -v;
        s.bce += (s.x[b] > 0.f ? 0.f : -s.x[b]) + log1pf(expf(-fabsf(s.x[b])));
    }
    s.right = expf(-s.bce);
    return s;
}

template <int M> __device__ __forceinline__ void write_grad(const LossArgs &a, int64_t image, int j, const Symbol<M> &s, float over)
{
    float *g = a.grad + image * a.n_bits + j * M;
    const float pull = a.per_bit + 2.f * a.per_image * over * s.right;
#pragma unroll
    for (int b = 0; b < M; ++b) {
        const float e = expf(-fabsf(s.x[b])), miss = (s.x[b] >= 0.f ? e : 1.f) / (1.f + e);
        g[b] = (s.ones >> b & 1 ? -miss : miss) * pull;
    }
}

// Sum over `lanes` neighbouring lanes, the same bits in each.
template <typename T> __device__ __forceinline__ T lanes_sum(T v, int lanes)
{
    for (int o = lanes / 2; o; o /= 2) v += __shfl_xor(v, o, 64);
    return v;
}

template <int M> __global__ __launch_bounds__(kSmallThreads) void message_loss_kernel(LossArgs a)
{
    __shared__ double sums[kSmallThreads / 64];
    const int lane = threadIdx.x & (a.lanes - 1), per = blockDim.x / a.lanes;
    double total = 0.0;
    // the loop is the same for all lanes of a wavefront: those of images past the last one compute nothing
    for (int64_t first = (int64_t)blockIdx.x * per; first < a.N; first += (int64_t)gridDim.x * per) {
        const int64_t image = first + threadIdx.x / a.lanes;
        const bool here = image < a.N;
        Symbol<M> mine; // this lane's first symbol stays, further ones (n > 64) are read again for the gradient
        float wrong = 0.f, bce = 0.f;
        int bits = 0, symbols = 0;
        if (here)
            for (int j = lane; j < a.n; j += a.lanes) {
                const Symbol<M> s = read_symbol<M>(a, image, j);
                if (j == lane) mine = s;
                wrong += 1.f - s.right;
                bce += s.bce;
                bits += s.wrong;
                symbols += s.wrong != 0;
            }
        wrong = lanes_sum(wrong, a.lanes);
        bce = lanes_sum(bce, a.lanes);
        bits = lanes_sum(bits, a.lanes);
        symbols = lanes_sum(symbols, a.lanes);
        const float excess = wrong - (float)a.t, over = a.weight > 0.f && !(excess <= 0.f) ? excess : 0.f;
        if (!here) continue;
        if (a.grad)
            for (int j = lane; j < a.n; j += a.lanes) write_grad<M>(a, image, j, j == lane ? mine : read_symbol<M>(a, image, j), over);
        if (lane == 0) {
            if (a.bit_errors) a.bit_errors[image] = bits;
            if (a.symbol_errors) a.symbol_errors[image] = symbols;
            total += (double)bce * a.per_bit + (double)over * over * a.per_image;
        }
    }
    total = lanes_sum(total, 64);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x / 64] = total;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < blockDim.x / 64; ++w) total += sums[w];
        if (a.partial) a.partial[blockIdx.x] = total;
        else *a.loss = (float)total;
    }
}

__global__ __launch_bounds__(256) void loss_sum_kernel(const double *partial, int count, float *loss)
{
    __shared__ double sums[4];
    double s = 0.0;
    for (int i = threadIdx.x; i < count; i += 256) s += partial[i];
    s = lanes_sum(s, 64);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x / 64] = s;
    __syncthreads();
    if (threadIdx.x == 0) *loss = (float)(sums[0] + sums[1] + sums[2] + sums[3]);
}

int lanes_of(int n)
{
    int lanes = 1;
    while (lanes < n && lanes < 64) lanes *= 2;
    return lanes;
}

} // namespace

// Workgroups of a call; one of 1024 threads up to four images a lane group, then no second launch is needed.
int64_t loss_blocks(int64_t N, int n)
{
    const int lanes = lanes_of(n);
    if (N <= 4 * (kSmallThreads / lanes)) return 1;
    return std::min<int64_t>((N + kThreads / lanes - 1) / (kThreads / lanes), 2048);
}

hipError_t launch_message_loss(const LossCall &c, double *partial, hipStream_t s)
{
    const int64_t blocks = loss_blocks(c.N, c.n);
    const double images = c.N ? (double)c.N : 1.0;
    LossArgs a{c.logits, c.target, c.target_stride, c.N, c.n_bits, c.n, c.t, lanes_of(c.n), c.weight, (float)(1.0 / (images * c.n_bits)),
               (float)(c.weight / images), c.loss, c.grad, c.bit_errors, c.symbol_errors, blocks > 1 ? partial : nullptr};
    const dim3 grid((uint32_t)blocks), block(blocks > 1 ? kThreads : kSmallThreads);
    auto run = [&](auto m) { hipLaunchKernelGGL((message_loss_kernel<decltype(m)::value>), grid, block, 0, s, a); };
    switch (c.m) {
    case 1: run(std::integral_constant<int, 1>()); break;
    case 2: run(std::integral_constant<int, 2>()); break;
    case 3: run(std::integral_constant<int, 3>()); break;
    case 4: run(std::integral_constant<int, 4>()); break;
    case 5: run(std::integral_constant<int, 5>()); break;
    case 6: run(std::integral_constant<int, 6>()); break;
    case 7: run(std::integral_constant<int, 7>()); break;
    default: run(std::integral_constant<int, 8>()); break;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || blocks == 1) return e;
    hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(256), 0, s, partial, (int)blocks, c.loss);
    return hipGetLastError();
}

} // namespace qrm
