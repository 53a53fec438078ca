// Group norm with an activation: how a call is cut into workgroups, and what does not depend on the element type (kernels: group_norm.h).
#include "qrm_train.h"

#include <algorithm>
#include <cmath>
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
    if (unit / p.V > kNormThreads) { // (pieces that straddle groups: the shared memory holds 256 of them; those that divide a group are no more)
        p.V = std::gcd(D, p.V);
        unit = D;
    }
    if (unit / p.V > kNormMaxThreads) return false; // D / gcd(D, V), whichever
    p.W = D % p.V == 0 ? 1 : p.V % D == 0 ? p.V / D : p.V;
    auto cut = [&](int bytes, int threads) { // whole groups, at least so many bytes wide
        NormCut c;
        c.ct = (int)std::min<int64_t>(d.C, (bytes + unit * size - 1) / (unit * size) * unit);
        c.tiles = (d.C + c.ct - 1) / c.ct;
        c.threads = std::max(threads, (c.ct / p.V + 63) / 64 * 64);
        c.chunks = 1;
        return c;
    };
    auto deal = [&](NormCut &c, int per_cu, int most) { // so many workgroups to a compute unit, if that leaves each four pixels a thread, and up to `most`
        const int rpar = c.threads / (c.ct / p.V);
        const int64_t want = std::max<int64_t>(1, (int64_t)per_cu * num_cu / std::max<int64_t>(1, d.N * c.tiles));
        c.chunks = (int)std::max(std::min(want, std::max<int64_t>(1, d.P / (4 * rpar))), (d.P - 1) / ((int64_t)most * rpar) + 1);
    };

    // A tile for one launch is the narrowest, down to 16 channels (8 forward), of which there are not more than compute units: a line's tiles are numbered so that one
    // die's cache serves them all (find_tile).  One launch is taken where a tile fits a workgroup and is over before a second launch would have begun, or
    // where compute units are busy anyway and the map is read once.  Measured with silu and 512 channels in bf16 on one map again and again, one launch / two, us: 1 image
    // of 256 / 1024 / 2048 pixels 6.3 / 9.7, 7.5 / 9.7, 10.1 / 9.9; 4 images of 1024 / 2048 / 4096 7.9 / 10.2, 11.1 / 12.2, 16.4 / 16.4 (tiles of a line, 1024 pixels: 12.8); 16 images
    // 11.7 / 16.3, 18.9 / 22.5, 28.8 / 34.6 (a line 14.7, 24.1); 64 images of 1024, on other maps in turn, 24.5 / 39.0; backward, 1 image of 256 / 1024 / 2048 pixels
    // 7.3 / 11.6, 8.4 / 11.6, 14.8 / 11.8; 4 images 9.1 / 11.7, 11.8 / 12.3, 18.7 / 15.4; 16 images of 512 / 1024 11.7 / 15.3, 18.3 / 20.2.
    // In f32 1 image of 1024 pixels 7.4 / 9.4, 4 of 2048 10.9 / 13.4, 16 of 2048 24.2 / 31.1, 64 of 1024 42.7 / 64.8; backward 1 of 1024 9.8 / 10.6, 16 and 64 of 256 9.7 / 11.9,
    // 21.4 / 28.5.  128 channels, bf16 4 of 2048 8.2 / 10.5, 64 of 1024 11.2 / 16.9, backward 19.8 / 20.6; 320 channels, ten a group, bf16 16 of 256 8.6 / 12.6, backward 11.4 / 14.3. In
    // f32 these last are the one family that the rule costs something: backward, 16 and 64 images of 256 pixels 12.0 / 11.4, 27.8 / 26.3.
    const int most_threads = p.W > 2 ? 256 : backward ? kNormMaxThreads / 2 : kNormMaxThreads;
    const int least = (backward ? 16 : 8) * size;
    auto fit = [&] { // pixels and threads of a tile
        const int cols = p.first.ct / p.V;
        auto threads_for = [&](int pixels) { return std::min<int64_t>(INT32_MAX, ((d.P + pixels - 1) / pixels * cols + 255) / 256 * 256); };
        p.pixels = threads_for(kNormFew) <= most_threads ? kNormFew : norm_many(backward, p.W);
        const int64_t threads = threads_for(p.pixels);
        p.first.threads = (int)threads;
        return threads <= most_threads && d.P <= p.pixels * (threads / cols);
    };
    auto rounds = [&] { // of workgroups that run at once
        const int64_t at_once = (int64_t)num_cu * std::max(1, (p.pixels == kNormFew ? 2 : 1) * kNormMaxThreads / p.first.threads); // (for their registers)
        return (double)(d.N * p.first.tiles) / at_once;
    };
    auto pays = [&] {
        const int64_t blocks = d.N * p.first.tiles, elements = d.P * p.first.ct;
        if (!fit()) return false;
        if (backward) return elements * size <= (blocks >= num_cu ? 65536 : 32768);
        return blocks >= num_cu || elements <= (blocks >= num_cu / 2 ? 32768 : 16384);
    };
    int bytes = 128;
    p.first = cut(bytes, 64);
    while (bytes / 2 >= least) {
        const NormCut half = cut(bytes / 2, 64);
        if (d.N * half.tiles > num_cu) break;
        p.first = half, bytes /= 2;
    }
    // (rounds have to be three quarters full: 48 images of 2048 pixels and 512 channels, one and a half rounds 55.9 us, two launches 57.3; 24 of 4096 76.0 and 56.0)
    p.whole = pays() && (rounds() <= 1.0 || rounds() >= 0.75 * std::ceil(rounds()));
    if (!p.whole && bytes / 2 >= least) { // a few more tiles than compute units, side by side: 20 images of 2048 pixels 25.0, two launches 26.7
        p.first = cut(bytes / 2, 64);
        p.whole = pays() && rounds() <= 1.0 && !(backward && d.P * p.first.ct * size > 32768);
    }
    if (!p.whole) {
        // (few chunks in the first launch: every workgroup of the second reads its groups' parts of all of them)
        p.first = p.second = cut(128, kNormThreads);
        deal(p.first, 2, kNormRow);
        deal(p.second, backward ? 2 : 4, INT32_MAX);
        p.part_words = (size_t)d.N * d.groups * p.first.chunks;
    }
    // Outputs larger than all L2s (8 x 4 MiB) are written past the caches: who reads them next finds little of them there, and what they would push out of the memory-side
    // cache is written to memory while the next launch reads.  4 images of 256 x 256 pixels, 128 channels, bf16 (64 MiB): 43.6 us without, 38.6 with;
    // backward 72.0 and 62.4; in one launch 64 images of 1024 pixels, 512 channels 37.8 and 24.5.  Parts of lines, from several workgroups, are better put together in the
    // caches: 16 images of 4096 pixels, 512 channels in f32, half lines, 71.7 without, 85.6 with.
    p.stream = (double)d.N * d.P * d.C * size > 32.0 * (1 << 20) && (!p.whole || p.first.ct * size >= 128);
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
