// Message loss with its gradient (qrm_message_loss).
//
// A lane takes a symbol, 2^k lanes an image: the image's expected number of wrong symbols, which every bit's gradient depends on, is a sum over
// neighbouring lanes.  Workgroups leave their part of the loss in 64 bits; the last one that is done adds them up, in their order.  Bound by latency: 4 images
// of 48 bits 2.5 us, a launch and one round of loads; 16384 of 96 bits (14 MB) 8.7 us, of which loads and arithmetic take 5 (a quarter of the lanes have no
// symbol), the rest counting the workgroups and adding their parts.  All 256 counted in one word: 10.5 us; workgroups of 512 or 256 threads: the same within 0.3.
#include "qrm_train.h"

#include <algorithm>
#include <type_traits>

namespace qrm {
namespace {

constexpr int kThreads = 1024;
constexpr int kSet = 16, kLine = 32; // workgroups that share a count; words from one count to the next

struct LossArgs {
    const float *logits;
    const uint8_t *target;
    int64_t target_stride, N;
    int n_bits, n, t, lanes; // lanes: of an image, a power of two
    float weight, per_bit, per_image; // 1 / (N n_bits), weight / N
    float *loss, *grad;
    int32_t *bit_errors, *symbol_errors;
    bool wide;       // logits and gradients lie on 16-byte boundaries
    double *partial; // [workgroups], unless there is only one
    uint32_t *done;  // workgroups that are; 0 between calls
};

template <int M> struct Symbol {
    float miss[M];     // chance that a bit is wrong
    uint32_t ones;     // target bits
    int wrong;         // hard bits that differ
    float bce, right;  // sum of -log sigmoid(x); chance that all bits are right
};

// sigmoid(x) and sigmoid(-x) of a symbol's bits from e = exp(-|x|) <= 1.
template <int M, bool FAR> __device__ __forceinline__ void chances(Symbol<M> &s, const float (&x)[M])
{
    s.bce = 0.f;
    s.right = 1.f;
#pragma unroll
    for (int b = 0; b < M; ++b) {
        const float e = FAR ? expf(-fabsf(x[b])) : __builtin_amdgcn_exp2f(fabsf(x[b]) * -1.44269504f), w = 1.f + e, r = __builtin_amdgcn_rcpf(w);
        const bool good = x[b] >= 0.f;
        const float q = e * r;
        s.miss[b] = good ? q : r;
        s.right *= good ? r : q;
        // log(1 + e): the logarithm of the rounded sum and, to first order, of what the rounding left out
        s.bce += fmaf(e - (w - 1.f), r, __builtin_amdgcn_logf(w) * 0.693147181f) + (x[b] > 0.f ? 0.f : -x[b]); // (a NaN stays one)
    }
}

template <int M> __device__ __forceinline__ Symbol<M> read_symbol(const LossArgs &a, int64_t image, int j)
{
    constexpr int V = M % 4 == 0 ? 4 : 1;
    Symbol<M> s;
    const float *z = a.logits + image * a.n_bits + j * M;
    const uint8_t *target = a.target + image * a.target_stride + j * M;
    float v[M];
#pragma unroll
    for (int b = 0; b < M; b += V) {
        if (V == 4 && a.wide) {
            const Pack<float, V> p = load_pack<float, V>(z + b);
#pragma unroll
            for (int k = 0; k < V; ++k) v[b + k] = p.e[k];
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k) v[b + k] = z[b + k];
        }
    }
    s.ones = 0;
    s.wrong = 0;
    float farthest = 0.f;
#pragma unroll
    for (int b = 0; b < M; ++b) {
        const bool one = target[b] != 0;
        s.ones |= (uint32_t)one << b;
        s.wrong += (v[b] > 0.f) != one;
        v[b] = one ? v[b] : -v[b]; // x = s * logit
        farthest = fmaxf(farthest, fabsf(v[b]));
    }
    // The hardware's functions are within 1 ulp, but know no numbers below 2^-126: symbols with a logit that far off take the library's.
    if (farthest < 80.f) chances<M, false>(s, v);
    else chances<M, true>(s, v);
    return s;
}

template <int M> __device__ __forceinline__ void write_grad(const LossArgs &a, int64_t image, int j, const Symbol<M> &s, float over)
{
    constexpr int V = M % 4 == 0 ? 4 : 1;
    float *g = a.grad + image * a.n_bits + j * M;
    const float pull = a.per_bit + 2.f * a.per_image * over * s.right;
#pragma unroll
    for (int b = 0; b < M; b += V) {
        Pack<float, V> p;
#pragma unroll
        for (int k = 0; k < V; ++k) p.e[k] = (s.ones >> (b + k) & 1 ? -pull : pull) * s.miss[b + k];
        if (V == 4 && a.wide) {
            store_pack<float, V>(g + b, p);
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k) g[b + k] = p.e[k];
        }
    }
}

// v plus that of another lane of the row of 16, which CTRL picks.
template <int CTRL, typename T> __device__ __forceinline__ T add_lane(T v)
{
    return v + __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// Sum over `lanes` neighbouring lanes, the same bits in each: pairs, fours, halves of a row and rows by lane moves in the vector unit.
template <typename T> __device__ __forceinline__ T lanes_sum(T v, int lanes)
{
    if (lanes > 1) v = add_lane<0xB1>(v);   // quad_perm [1,0,3,2]
    if (lanes > 2) v = add_lane<0x4E>(v);   // quad_perm [2,3,0,1]
    if (lanes > 4) v = add_lane<0x141>(v);  // row_half_mirror
    if (lanes > 8) v = add_lane<0x140>(v);  // row_mirror
    if (lanes > 16) v += __shfl_xor(v, 16);
    if (lanes > 32) v += __shfl_xor(v, 32);
    return v;
}
// A barrier for shared memory alone: stores to memory may be under way.
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <int M> __global__ __launch_bounds__(kThreads) void message_loss_kernel(LossArgs a)
{
    __shared__ double sums[kThreads / 64];
    __shared__ bool last;
    const int lane = threadIdx.x & (a.lanes - 1), per = blockDim.x / a.lanes;
    double total = 0.0;
    Symbol<M> mine; // this lane's first symbol stays, further ones (n > 64) are read again for the gradient
    float over = 0.f;
    int64_t image = a.N;
    auto write_image = [&] {
        if (a.grad && image < a.N)
            for (int j = lane; j < a.n; j += a.lanes) write_grad<M>(a, image, j, j == lane ? mine : read_symbol<M>(a, image, j), over);
    };
    // the loop is the same for all lanes of a wavefront: those of images past the last one compute nothing
    for (int64_t first = (int64_t)blockIdx.x * per; first < a.N; first += (int64_t)gridDim.x * per) {
        write_image(); // the last round's: this round's waits until the part of the loss is on its way
        image = first + threadIdx.x / a.lanes;
        const bool here = image < a.N;
        float wrong = 0.f, bce = 0.f;
        int errors = 0; // bits, and in the upper half symbols
        if (here)
            for (int j = lane; j < a.n; j += a.lanes) {
                const Symbol<M> s = read_symbol<M>(a, image, j);
                if (j == lane) mine = s;
                wrong += 1.f - s.right;
                bce += s.bce;
                errors += s.wrong + (s.wrong ? 0x10000 : 0);
            }
        wrong = lanes_sum(wrong, a.lanes);
        bce = lanes_sum(bce, a.lanes);
        errors = lanes_sum(errors, a.lanes);
        const float excess = wrong - (float)a.t;
        over = a.weight > 0.f && !(excess <= 0.f) ? excess : 0.f;
        if (here && lane == 0) {
            if (a.bit_errors) a.bit_errors[image] = errors & 0xffff;
            if (a.symbol_errors) a.symbol_errors[image] = errors >> 16;
            total += (double)bce * a.per_bit + (double)over * over * a.per_image;
        }
    }
    auto add_up = [&](double v, int apart) { // over the workgroup, of lanes `apart`; thread 0 has the sum
        for (int o = 32; o >= apart; o /= 2) v += __shfl_down(v, o);
        if (blockDim.x == 64) return v;
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x / 64] = v;
        lds_barrier();
        if (threadIdx.x == 0)
            for (int w = 1; w < (int)blockDim.x / 64; ++w) v += sums[w];
        return v;
    };
    total = add_up(total, a.lanes);
    if (gridDim.x == 1) {
        if (threadIdx.x == 0) *a.loss = (float)total;
        write_image();
        return;
    }
    // parts and count are stored past the L2s; a part has arrived before its workgroup is counted
    if (threadIdx.x == 0) {
        __hip_atomic_store(a.partial + blockIdx.x, total, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        // (additions to one word follow each other: sixteen workgroups share one, in a line of its own, and the last of them counts on in the first word)
        const auto counted = [](uint32_t *word, uint32_t all) {
            const bool full = __hip_atomic_fetch_add(word, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == all;
            if (full) __hip_atomic_store(word, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            return full;
        };
        const uint32_t sets = (gridDim.x + kSet - 1) / kSet, set = blockIdx.x % sets;
        last = counted(a.done + (1 + set) * kLine, gridDim.x / sets + (set < gridDim.x % sets)) && counted(a.done, sets);
    }
    write_image();
    lds_barrier();
    if (!last) return;
    total = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += blockDim.x) total += __hip_atomic_load(a.partial + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    total = add_up(total, 1);
    if (threadIdx.x == 0) *a.loss = (float)total;
}

int lanes_of(int n)
{
    int lanes = 1;
    while (lanes < n && lanes < 64) lanes *= 2;
    return lanes;
}

} // namespace

// Workgroups of a call: one for up to four images a lane group of 1024 threads, else at most 256: one to a compute unit.
int64_t loss_blocks(int64_t N, int n)
{
    const int64_t per = kThreads / lanes_of(n);
    return N <= 4 * per ? 1 : std::min<int64_t>((N + per - 1) / per, 256);
}

hipError_t launch_message_loss(const LossCall &c, double *partial, uint32_t *done, hipStream_t s)
{
    const int64_t blocks = loss_blocks(c.N, c.n);
    const double images = c.N ? (double)c.N : 1.0;
    const int lanes = lanes_of(c.n);
    const bool wide = ((uintptr_t)c.logits | (uintptr_t)c.grad) % 16 == 0;
    LossArgs a{c.logits, c.target, c.target_stride, c.N, c.n_bits, c.n, c.t, lanes, c.weight, (float)(1.0 / (images * c.n_bits)),
               (float)(c.weight / images), c.loss, c.grad, c.bit_errors, c.symbol_errors, wide, partial, done};
    const dim3 grid((uint32_t)blocks), block(blocks > 1 ? kThreads : (int)std::min<int64_t>(kThreads, std::max<int64_t>(1, (c.N * lanes + 63) / 64) * 64));
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
    return hipGetLastError();
}

} // namespace qrm
