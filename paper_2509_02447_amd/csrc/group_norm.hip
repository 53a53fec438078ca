// Group norm with an activation: how a call is cut into workgroups, and what does not depend on the element type (kernels: group_norm.h).
#include "qrm_train.h"

#include <algorithm>
#include <numeric>

namespace qrm {
namespace {

// Zeros for dgamma and dbeta of no images.
__global__ void norm_zero_kernel(float *dgamma, float *dbeta, int C)
{
    const int c = blockIdx.x * blockDim.x + threadIdx.x;
    if (c < C && dgamma) dgamma[c] = 0.f;
    if (c < C && dbeta) dbeta[c] = 0.f;
}

} // namespace

bool plan_norm(const qrm_group_norm_desc &d, int align_bytes, bool backward, bool channels, int num_cu, NormPlan *out)
{
    const int size = type_bytes(d.type), D = d.C / d.groups;
    NormPlan p{};
    // the widest piece that the addresses, the strides and the number of channels allow
    p.V = std::min(16, align_bytes) / size;
    while (d.C % p.V || d.x_pixel % p.V || d.y_pixel % p.V || d.x_image % p.V || d.y_image % p.V) p.V /= 2;
    int64_t unit = std::lcm<int64_t>(D, p.V);
    if (unit / p.V > kNormThreads) { // (pieces that straddle groups: the shared memory holds 256 of them)
        p.V = std::gcd(D, p.V);
        unit = D;
    }
    if (unit / p.V > kNormMaxThreads) return false;
    p.W = D % p.V == 0 ? 1 : p.V % D == 0 ? p.V / D : p.V;
    auto cut = [&](int bytes, int threads) { // whole groups, at least so many bytes wide
        NormCut c;
        c.ct = (int)std::min<int64_t>(d.C, (bytes + unit * size - 1) / (unit * size) * unit);
        c.tiles = (d.C + c.ct - 1) / c.ct;
        c.threads = std::max(threads, (c.ct / p.V + 63) / 64 * 64);
        c.chunks = 1;
        return c;
    };
    auto deal = [&](NormCut &c, int per_cu) { // so many workgroups to a compute unit, if that leaves each four pixels a thread
        const int rpar = c.threads / (c.ct / p.V);
        const int64_t want = std::max<int64_t>(1, (int64_t)per_cu * num_cu / std::max<int64_t>(1, d.N * c.tiles));
        c.chunks = (int)std::min(want, std::max<int64_t>(1, d.P / (4 * rpar)));
    };

    // One launch where a tile of an image fits a workgroup, if that is over before a second launch would have begun or keeps all compute units
    // busy.  Where tiles of a line leave compute units idle, they are half a line wide, and a quarter where there are very few (narrow ones share their lines
    // with other dies' caches).  Measured with silu and bf16, one launch / two, us: 1 image of 512 channels, 64 / 256 / 1024 / 2048 pixels 5.7 / 9.3,
    // 5.7 / 9.7, 7.4 / 9.8, 10.1 / 9.9; 4 images of 256 / 1024 / 2048 pixels 6.0 / 9.9, 9.6 / 10.3, 13.4 / 12.3; 16 of 1024 13.6 / 16.4; 32 of 2048
    // 27.7 / 38.5; backward, 1 image, 256 / 1024 / 2048 pixels 7.0 / 11.5, 11.1 / 11.6, 18.7 / 11.8; 4 of 256 / 512 / 1024 9.6 / 11.7, 11.7 / 11.8, 18.0 / 12.3.
    const int most_threads = p.W > 2 ? 256 : backward ? kNormMaxThreads / 2 : kNormMaxThreads;
    p.first = cut(128, 64);
    const bool many_tiles = d.N * p.first.tiles >= num_cu;
    if (!many_tiles) {
        const NormCut half = cut(64, 64), quarter = cut(32, 64);
        if (d.N * quarter.tiles <= num_cu / 4) p.first = quarter;
        else if (d.N * half.tiles <= num_cu) p.first = half;
    }
    const int64_t most = backward || p.first.ct * size < 64 ? 16384 : 32768; // elements of a tile
    const int cols = p.first.ct / p.V;
    auto threads_for = [&](int pixels) { return std::min<int64_t>(INT32_MAX, ((d.P + pixels - 1) / pixels * cols + 255) / 256 * 256); };
    p.pixels = threads_for(kNormFew) <= most_threads ? kNormFew : norm_many(backward, p.W);
    const int64_t threads = threads_for(p.pixels);
    p.whole = threads <= most_threads && d.P <= p.pixels * (threads / cols) &&
              (many_tiles || (d.P * p.first.ct <= most && !(backward && d.N > 1 && d.P > 512)));
    if (p.whole) {
        p.first.threads = (int)threads;
        p.part_words = 0;
    } else {
        // (few chunks in the first launch: every workgroup of the second reads its groups' parts of all of them)
        p.first = p.second = cut(128, kNormThreads);
        deal(p.first, 2);
        deal(p.second, backward ? 2 : 4);
        p.part_words = (size_t)d.N * d.groups * p.first.chunks;
    }
    // Outputs larger than all L2s (8 x 4 MiB) are written past the caches: who reads them next finds little of them there, and what they would push out of the memory-side
    // cache is written to memory while the next launch reads.  4 images of 256 x 256 pixels, 128 channels, bf16 (64 MiB): 43.6 us without, 38.6 with;
    // backward 72.0 and 62.4.
    p.stream = (double)d.N * d.P * d.C * size > 32.0 * (1 << 20);
    p.channels = backward && channels && !(p.whole && d.N == 1);
    p.bytes = (p.part_words + (p.channels ? (size_t)d.N * p.first.chunks * d.C : 0)) * sizeof(float2);
    *out = p;
    return true;
}

#define QRM_NORM_TYPE(NAME)                                                                                \
    hipError_t launch_norm_forward_##NAME(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s);  \
    hipError_t launch_norm_backward_##NAME(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s);
QRM_NORM_TYPE(f32)
QRM_NORM_TYPE(bf16)
QRM_NORM_TYPE(f16)
#undef QRM_NORM_TYPE

hipError_t launch_norm_forward(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s)
{
    return c.d.type == QRM_F32 ? launch_norm_forward_f32(c, p, ws, s)
           : c.d.type == QRM_BF16 ? launch_norm_forward_bf16(c, p, ws, s) : launch_norm_forward_f16(c, p, ws, s);
}

hipError_t launch_norm_backward(const NormCall &c, const NormPlan &p, void *ws, hipStream_t s)
{
    if (c.d.N == 0) {
        hipLaunchKernelGGL(norm_zero_kernel, dim3((c.d.C + 255) / 256), dim3(256), 0, s, c.dgamma, c.dbeta, c.d.C);
        return hipGetLastError();
    }
    return c.d.type == QRM_F32 ? launch_norm_backward_f32(c, p, ws, s)
           : c.d.type == QRM_BF16 ? launch_norm_backward_bf16(c, p, ws, s) : launch_norm_backward_f16(c, p, ws, s);
}

} // namespace qrm
