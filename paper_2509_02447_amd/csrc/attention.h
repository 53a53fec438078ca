// Attention over the rows of a map, forward and backward (qrm_attention, qrm_attention_backward): kernels, for one element type a source file.
//
// A column of matrix products belongs to a lane.  A wavefront holds M query rows (backward for keys: M key rows) as columns and walks down the other side's
// rows in tiles that lie in LDS as they lie in memory.  Scores are computed with those rows as the products' rows, so that a lane has the scores of its
// own column: maxima and sums stay in the lane but for one or two lane exchanges, and the scores go back into the next product as its column operand
// without leaving their registers: the order of the summed index is the same on both sides, whichever it is (kappa below).  The other operand of that
// product is the tile again, transposed by the LDS read.
//
// Rows of 1 KB and more would not leave the registers two wavefronts to a SIMD.  There two wavefronts share a set of columns: each has half of the elements of
// the rows and of the results, computes half of every score's sum, and they exchange these halves through LDS.
//
// Heads that share keys: query rows are counted (position, head of the group), so a tile of keys is read once for all of them; gradients of shared keys
// are summed over the group inside one workgroup.  No atomics anywhere: the backward pass computes the scores twice, once with queries as columns for dq
// and once with keys as columns for dk and dv.
#pragma once

#include "qrm_train.h"

namespace qrm {

typedef __attribute__((address_space(3))) uint8_t *lds_t;

// Products of M x 8 NG by 8 NG x M: `a` has row lane % M, `b` column lane % M, both elements 8 g + j of the summed index, g = lane / M.  The result's
// column is lane % M, its rows those of row_of.
template <typename T, int M> struct Mma {
    static constexpr int NG = 64 / M, KK = 8 * NG, C = M * M / 64;
    typedef T frag __attribute__((ext_vector_type(8)));
    typedef float acc __attribute__((ext_vector_type(C)));
    static __device__ __forceinline__ acc mul(frag a, frag b, acc c)
    {
        if constexpr (std::is_same<T, bf16_t>::value) {
            if constexpr (M == 32) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
            else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
        } else if constexpr (std::is_same<T, f16_t>::value) {
            if constexpr (M == 32) return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
            else return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) { // (any order of the summed index will do, as long as both sides have it)
                if constexpr (M == 32) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
                else c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
            }
            return c;
        }
    }
    // Row of a lane's r-th result where blocks of M rows lie one below the other; also the summed index of element r % 8 of the r / 8 -th column operand
    // that is made of them.
    static __device__ __forceinline__ int row_of(int r, int g) { return r / 4 * (4 * NG) + 4 * g + r % 4; }
};

// A wavefront's load of 64 times 16 (4) bytes, at off (per lane) of the resource, to `to` and what follows.  In asm, so that the compiler, which cannot tell
// the tiles apart, does not wait for the next one before every read of this one; whoever reads waits (wait_loads) and passes a barrier.  (m0 holds nothing
// else in these kernels: it is set where it is used.)
__device__ __forceinline__ void load_to_lds16(__amdgpu_buffer_rsrc_t rsrc, uint32_t off, uint8_t *to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"((uint32_t)(uintptr_t)(lds_t)to), "v"(off), "s"(rsrc) : "memory");
}
__device__ __forceinline__ void load_to_lds4(__amdgpu_buffer_rsrc_t rsrc, uint32_t off, uint8_t *to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"((uint32_t)(uintptr_t)(lds_t)to), "v"(off), "s"(rsrc) : "memory");
}
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// .. of the loads that the compiler knows: said once before a loop, it does not wait for them inside, and for what is under way there.
__device__ __forceinline__ void wait_known_loads() { __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8)); }

__device__ __forceinline__ uint32_t again_scalar(uint32_t v)
{
    asm volatile("" : "+s"(v));
    return v;
}
// A value that what follows is computed from anew, instead of being kept in registers from before.
__device__ __forceinline__ int again(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// A tile in LDS: rows of PB bytes, a power of two, whose pieces of 16 bytes are swapped about within the row (swizzle) so that neither the reads of one
// piece of 16 neighbouring rows nor those of 4 rows by 4 pieces meet in one of the 64 banks.
template <typename T, int DP> struct Tile {
    static constexpr int PB = attn_pitch(DP * (int)sizeof(T)), E = 16 / (int)sizeof(T), PIECES = PB / 16;
    static __device__ __forceinline__ int swizzle(int row)
    {
        const int four = (row >> 2 & 3) ^ (row >> 2 & 1) << 1; // 0, 3, 2, 1
        return PB == 128 ? (row >> 1 & 1) << 2 | four : (row & 3) << 2 | four;
    }

    // Rows 0 .. ROWS-1 of `src` (row_bytes apart, `rows` of them there, D elements each) on their way into the tile; what is not there becomes zeros.
    // WAVES * 64 threads; everything lies on 16 bytes.
    template <int ROWS, int WAVES>
    static __device__ __forceinline__ void load(const uint8_t *src, int row_bytes, int rows, int D, uint8_t *tile, int tid, int wave)
    {
        constexpr int COUNT = ROWS * PIECES;
        static_assert(COUNT % (WAVES * 64) == 0, "whole wavefronts load a tile");
        rows = max(0, min(rows, ROWS));
        const int bytes = rows ? (rows - 1) * row_bytes + D * (int)sizeof(T) : 0;
        __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(src), 0, bytes, 0x00020000);
        // A lane's loads are APART rows apart; the swizzle of a sum of rows without common bits is that of the one and that of the other.  Offsets are computed anew
        // each time, two instructions each: kept, they would take a register each.
        constexpr int APART = WAVES * 64 / PIECES;
        asm volatile("" : "+s"(row_bytes));
        const int row = tid / PIECES, piece = (tid % PIECES) ^ swizzle(row), start = __mul24(row, row_bytes);
        const bool full = D == PB / (int)sizeof(T);
#pragma unroll
        for (int k = 0; k < COUNT / (WAVES * 64); ++k) {
            const int p = piece ^ swizzle(k * APART);
            uint32_t off = start + k * APART * row_bytes + p * 16;
            if (!full) off = p * E < D ? off : 0x80000000u;
            load_to_lds16(rsrc, off, tile + (k * WAVES + wave) * 1024);
        }
    }

    // An LDS address of a tile's operand is one address of the lane, whose piece is changed by a constant, plus a constant: MASK is what the swizzle reaches.
    static constexpr int MASK = PB == 128 ? 7 : 15;
    static __device__ __forceinline__ uint32_t piece_at(uint32_t at, int piece, int add) { return (at ^ (uint32_t)(piece & MASK) << 4) + (uint32_t)((piece & ~MASK) * 16 + add); }
    template <typename V> static __device__ __forceinline__ void write(uint32_t at, V v) { *(__attribute__((address_space(3))) V *)(uintptr_t)at = v; }
    template <typename V> static __device__ __forceinline__ V read(uint32_t at) { return *(const __attribute__((address_space(3))) V *)(uintptr_t)at; }

    // Row operand of a product that sums over the row's elements, steps of 8 NG: the lane's address for row `row` of the tile, and the operand of a
    // step from the tile and the block of 16 rows (or a multiple) that lie `add` bytes behind.
    template <int M> static __device__ __forceinline__ uint32_t along_at(int row, int g) { return row * PB + (((sizeof(T) / 2 * g) ^ swizzle(row)) << 4); }
    template <int M> static __device__ __forceinline__ typename Mma<T, M>::frag along(uint32_t at, int step, int add)
    {
        typedef typename Mma<T, M>::frag frag;
        if constexpr (sizeof(T) == 2) {
            return read<frag>(piece_at(at, step * Mma<T, M>::NG, add));
        } else {
            const f32x4 lo = read<f32x4>(piece_at(at, 2 * step * Mma<T, M>::NG, add)), hi = read<f32x4>(piece_at(at, 2 * step * Mma<T, M>::NG + 1, add));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }

    // Row operand of a product that sums over the tile's rows: its rows are elements d0 .. d0 + M - 1, element j of the summed index tile row
    // first + row_of(j, g), `first` a multiple of 8 NG.  16-bit types: 16 lanes read 4 rows of 16 elements and hold 16 columns of 4.
    template <int M> static __device__ __forceinline__ uint32_t across_at(int lane)
    {
        const int g = lane / M, row = 4 * g + (sizeof(T) == 2 ? lane % 16 / 4 : 0);
        if (sizeof(T) == 2) return row * PB + (((lane % M / 16 * 2 + lane % 4 / 2) ^ swizzle(row)) << 4) + lane % 2 * 8;
        return row * PB + ((lane % M / 4 ^ swizzle(row)) << 4) + lane % 4 * 4;
    }
    template <int M> static __device__ __forceinline__ typename Mma<T, M>::frag across(uint32_t at, int first, int d0, int add)
    {
        typedef Mma<T, M> X;
        typedef typename X::frag frag;
        if constexpr (sizeof(T) == 2) {
            typedef short v4 __attribute__((ext_vector_type(4)));
            typedef short v8 __attribute__((ext_vector_type(8)));
            v4 part[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) { // (eight rows further on the swizzle is another by 2, sixteen further on the same)
                const uint32_t from = piece_at(at, d0 / 8 ^ (M == 32 ? 2 * u : 0), (first + u * 4 * X::NG) * PB + add);
                part[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4 *)(uintptr_t)from);
            }
            return __builtin_bit_cast(frag, (v8)__builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            frag f;
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = read<float>(piece_at(at, d0 / 4 ^ swizzle(j % 4) ^ (M == 32 ? j / 4 * 2 : 0), (first + X::row_of(j, 0)) * PB + add));
            return f;
        }
    }
};

// Eight elements of a row in memory from d on, zeros behind its end.
template <typename T> __device__ __forceinline__ auto row_piece(const T *row, bool there, int d, int D)
{
    typedef T frag __attribute__((ext_vector_type(8)));
    constexpr int E = 16 / (int)sizeof(T);
    frag f = {};
#pragma unroll
    for (int h = 0; h < 8 / E; ++h)
        if (there && d + h * E < D) {
            const Pack<T, E> v = load_pack<T, E>(row + d + h * E);
#pragma unroll
            for (int e = 0; e < E; ++e) f[h * E + e] = v.e[e];
        }
    return f;
}

// Four results of a row, from element d on.
template <typename T> __device__ __forceinline__ void store_four(T *row, int d, int D, float a, float b, float c, float e)
{
    if (d < D) store_pack<T, 4>(row + d, Pack<T, 4>{{(T)a, (T)b, (T)c, (T)e}});
}

// The barrier leaves loads into the other tile under way: it waits for lgkmcnt alone.
constexpr int kAttnWaitLds = 15 | (3 << 14) | (7 << 4);
__device__ __forceinline__ void attn_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(kAttnWaitLds);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// f32: an operand's eight loads are not on their way before the operand before it has been used, or there would be no registers for the sums; its eight products
// take 256 cycles and more.
template <typename T> __device__ __forceinline__ void one_by_one()
{
    if (sizeof(T) == 4) __builtin_amdgcn_sched_barrier(0);
}

// Order of a block of COUNT turns of PRODUCTS products with READS LDS reads together (and FIRST reads before them): the reads of AHEAD turns are on their way
// before the first product, and each turn's products are followed by the reads of another.  Left to itself the compiler reads just ahead of the use, and the products wait.
template <typename T, int COUNT, int READS, int AHEAD, int FIRST = 0, int PRODUCTS = 1> __device__ __forceinline__ void in_turn()
{
    if (sizeof(T) == 4) return;
    constexpr int DS = 0x100, MFMA = 0x8, A = AHEAD < COUNT ? AHEAD : COUNT;
    __builtin_amdgcn_sched_group_barrier(DS, FIRST + A * READS, 0);
#pragma unroll
    for (int i = 0; i < COUNT - A; ++i) {
        __builtin_amdgcn_sched_group_barrier(MFMA, PRODUCTS, 0);
        __builtin_amdgcn_sched_group_barrier(DS, READS, 0);
    }
    __builtin_amdgcn_sched_group_barrier(MFMA, A * PRODUCTS, 0);
}

// Eight numbers as a column operand: 16-bit types two to an instruction.
template <typename T> __device__ __forceinline__ auto pack_eight(const float *v)
{
    typedef T frag __attribute__((ext_vector_type(8)));
    if constexpr (sizeof(T) == 4) {
        return frag{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
    } else {
        typedef T pair __attribute__((ext_vector_type(2)));
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, (pair){(T)v[2 * i], (T)v[2 * i + 1]});
        return __builtin_bit_cast(frag, w);
    }
}

// Largest and sum over the lanes of a column.
template <int M> __device__ __forceinline__ float column_max(float v)
{
    if (M == 16) v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
template <int M> __device__ __forceinline__ float column_sum(float v)
{
    if (M == 16) v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

constexpr float kLog2E = 1.44269504088896341f;

// Where a workgroup is.  Workgroups that walk down the same keys are on one die, whose cache then serves them all, where there are eight groups of heads that
// share keys and more (consecutive workgroups are dealt to the eight dies in turn), or a number of them that divides eight; of a group's, those of one split
// follow each other.  false: behind the last one.
struct AttnPlace {
    int n, kv, part, split; // image, key head, tile of rows, split of the other side
};
__device__ __forceinline__ bool attn_place(const AttnArgs &a, int b, AttnPlace *p)
{
    const int per = a.parts * a.splits, groups = a.N * a.kv_heads;
    int group, rest;
    if (groups < 8 && (groups & (groups - 1)) == 0) {
        const int bits = __builtin_ctz(groups);
        group = b & (groups - 1);
        rest = (b >> 3 << (3 - bits)) + ((b & 7) >> bits);
        if (rest >= per) return false;
    } else {
        if (groups >= 8) b = (b & 7) * ((groups * per + 7) >> 3) + (b >> 3);
        if (b >= groups * per) return false;
        group = a.by_blocks.of(b);
        rest = b - group * per;
    }
    p->n = a.by_kv_heads.of(group);
    p->kv = group - p->n * a.kv_heads;
    p->split = a.by_parts.of(rest);
    p->part = rest - p->split * a.parts;
    return true;
}

// Where a split's results wait for those of others: as the lanes hold them, four results of a lane beside those of the next lane, so that a wavefront
// writes and reads 1 KB at a time.  attention_join_kernel knows which row's they are.
__device__ __forceinline__ int64_t attn_slot(const AttnArgs &a, const AttnPlace &at)
{
    return ((int64_t)at.split * a.N * a.kv_heads + at.n * a.kv_heads + at.kv) * a.parts + at.part;
}
template <int M, int WAVES, typename ACC, int COUNT> __device__ __forceinline__ void store_part(float *part, int64_t slot, int wave, int lane, float by, const ACC (&sums)[COUNT])
{
    constexpr int QUADS = M * M / 256;
    f32x4 *const to = (f32x4 *)part + ((slot * WAVES + wave) * COUNT * QUADS) * 64 + lane;
#pragma unroll
    for (int d = 0; d < COUNT; ++d)
#pragma unroll
        for (int r = 0; r < QUADS; ++r) to[(d * QUADS + r) * 64] = f32x4{sums[d][4 * r] * by, sums[d][4 * r + 1] * by, sums[d][4 * r + 2] * by, sums[d][4 * r + 3] * by};
}

// ---------------------------------------------------------------- forward

// Columns: query rows (position, head of the group).  Walks over the keys with a running maximum; the results are scaled down when it has grown by more
// than 2^GROWS, so that most tiles leave them alone.  Sums and results in 32 bits; probabilities are rounded to the type for the second product (16-bit types:
// half a step relative to each, unsystematic, which is what the output's own rounding is).  f16: they are taken times 2^11, so that many keys of little weight
// are not lost under its smallest number: 2^-36 a key (they stay under 2^16, with what the maximum may grow).
// Bound (kernels by a trace's medians; calls in a row without the profiler take less): rows of 128 and less, bf16, by the matrix pipe at the clock that the card's power allows (2 x 8192
// causal rows of 16 heads of 128: 545 us, 1.01 PFLOP/s, the call in a row 519, 1.06, where a large library product reaches 1.12); f32 by its products (3 x 2257 rows of 6 heads of 60: 225 us,
// 104 TFLOP/s counting the 64 elements that are computed); one head of 512 by LDS reads, which sixteen columns to a wavefront make twice what the products take (4 x 4096 rows: 179 us,
// 0.77 PFLOP/s, the call with its join 168 in a row; when two wavefronts shared 32 columns, which halves the reads, they waited for each other: calls of 184 against 164); single tokens by memory
// (16 over up to 8191 rows: 38 us, 4.3 TB/s of the keys and values that are there).
template <typename T, int DP, int M, int WAVES, int SHARE, int TK, int NBUF, int OCC>
__global__ __launch_bounds__(WAVES * 64, OCC) void attention_kernel(AttnArgs a)
{
    typedef Mma<T, M> X;
    typedef Tile<T, DP> L;
    constexpr int R = TK / X::NG, DH = DP / SHARE, AHEAD = 6; // scores of a lane, elements of a wavefront
    constexpr int TILES = NBUF * 2 * TK * L::PB, SWAP = R * 256; // exchanged: a wavefront's scores
    constexpr float GROWS = std::is_same<T, f16_t>::value ? 4.f : 8.f, LIFT = attn_lift(std::is_same<T, f16_t>::value), FAR = 0x1p14f;
    constexpr bool TURNS = NBUF == 1; // keys and values take turns: the one is on its way while the other is used
    static_assert(SHARE > 1 || !TURNS, "in turns there is a barrier between keys and values");
    __shared__ alignas(256) uint8_t lds[TILES + (SHARE > 1 ? WAVES * SWAP : 0)];
    AttnPlace at;
    if (!attn_place(a, blockIdx.x, &at)) return;
    if (a.causal) at.part = a.parts - 1 - at.part; // (the longest first)
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64), col = lane % M, g = lane / M;
    const int q_len = attn_length(a.q_len, at.n, a.Lq), k_len = attn_length(a.k_len, at.n, a.Lk), off = k_len - q_len;
    const int half = SHARE > 1 ? wave % SHARE : 0, e0 = half * DH; // which elements
    const int row0 = (at.part * (WAVES / SHARE) + wave / SHARE) * M, rows = a.Lq * a.group;
    int row = row0 + col, pos = attn_position(a, row), head = at.kv * a.group + (row - pos * a.group);
    const bool there = row < rows && pos < q_len;
    const int seen = there ? (a.causal ? max(0, min(k_len, pos + off + 1)) : k_len) : 0; // keys that the column sees
    // .. and the most and the least in the wavefront
    auto last_seen = [&](int last_row) { const int p = attn_position(a, min(last_row, rows - 1)); return a.causal ? max(0, min(k_len, min(p, q_len - 1) + off + 1)) : k_len; };
    const bool any = row0 < rows && attn_position(a, row0) < q_len;
    const int most = any ? last_seen(row0 + M - 1) : 0;
    const int least = row0 + M <= rows && attn_position(a, row0 + M - 1) < q_len ? (a.causal ? max(0, min(k_len, attn_position(a, row0) + off + 1)) : k_len) : 0;
    const AttnSplit split = attn_split(a, attn_key_tiles(a, q_len, k_len, at.part), at.split);
    if (at.split >= split.count) return;
    const int from = split.from, to = split.to;

    const uint8_t *const k = (const uint8_t *)a.k + (at.n * a.k_image + at.kv * a.k_head) * (int64_t)sizeof(T);
    const uint8_t *const v = (const uint8_t *)a.v + (at.n * a.v_image + at.kv * a.v_head) * (int64_t)sizeof(T);
    const int k_bytes = (int)a.k_row * (int)sizeof(T), v_bytes = (int)a.v_row * (int)sizeof(T);
    auto load_k = [&](int t) {
        L::template load<TK, WAVES>(k + (int64_t)t * TK * k_bytes, k_bytes, k_len - t * TK, a.D, lds + (t - from) % NBUF * (2 * TK * L::PB), tid, wave);
    };
    auto load_v = [&](int t) {
        L::template load<TK, WAVES>(v + (int64_t)t * TK * v_bytes, v_bytes, k_len - t * TK, a.D, lds + (t - from) % NBUF * (2 * TK * L::PB) + TK * L::PB, tid, wave);
    };
    if (from < to) {
        load_k(from);
        if (!TURNS) load_v(from);
    }

    typename X::frag q[DH / X::KK];
    const T *const q_row = (const T *)a.q + at.n * a.q_image + pos * a.q_row + head * a.q_head;
#pragma unroll
    for (int s = 0; s < DH / X::KK; ++s) q[s] = row_piece<T>(q_row, there, e0 + s * X::KK + 8 * g, a.D);

    typename X::acc o[DH / M] = {};
    wait_known_loads();
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_t)lds, mine = lds0 + e0 * (int)sizeof(T);
    const uint32_t along0 = mine + L::template along_at<M>(col, g), across0 = mine + L::template across_at<M>(lane);
    float top = -INFINITY, limit = -INFINITY, sums[4] = {}; // of the raw scores; what is 2^GROWS times as likely; of this lane's probabilities
    const float c = a.scale * kLog2E, grows = 0.999f * GROWS * __builtin_amdgcn_rcpf(c);
    bool far = false; // of the wavefront
    for (int t = from; t < to; ++t) {
        wait_loads();
        attn_barrier();
        if (TURNS) {
            load_v(t);
        } else if (t + 1 < to) {
            load_k(t + 1);
            load_v(t + 1);
        }
        const uint32_t tile = (t - from) % NBUF * (2 * TK * L::PB), along = along0 + tile, across = across0 + tile; // keys; values behind them
        const int first = t * TK;
        if (SHARE > 1 || first < most) { // (wavefronts that exchange halves wait for each other)
            typename X::acc s[TK / M];
#pragma unroll
            for (int b = 0; b < TK / M; ++b) s[b] = typename X::acc{};
#pragma unroll
            for (int i = 0; i < DH / X::KK; ++i)
#pragma unroll
                for (int b = 0; b < TK / M; ++b) { // (one after the other on other sums)
                    s[b] = X::mul(L::template along<M>(along, i, b * M * L::PB), q[i], s[b]);
                    one_by_one<T>();
                }
            in_turn<T, TK / M * (DH / X::KK), 1, AHEAD>();
            if constexpr (SHARE > 1) {
                const uint32_t to_other = lds0 + TILES + wave * SWAP + lane * 16, from_other = lds0 + TILES + (wave ^ 1) * SWAP + lane * 16;
#pragma unroll
                for (int r = 0; r < R; r += 4) L::write(to_other + r * 256, f32x4{s[r / X::C][r % X::C], s[r / X::C][r % X::C + 1], s[r / X::C][r % X::C + 2], s[r / X::C][r % X::C + 3]});
                if (TURNS) wait_loads(); // the values are there
                attn_barrier();          // .. everybody's, and everybody has read the keys
                if (TURNS && t + 1 < to) load_k(t + 1);
#pragma unroll
                for (int r = 0; r < R; r += 4) {
                    const f32x4 other = L::template read<f32x4>(from_other + r * 256);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[r / X::C][r % X::C + e] += other[e];
                }
            }
            auto score = [&](int r) -> float { return s[r / X::C][r % X::C]; };
            if (first + TK > least) {
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (first + X::row_of(r, g) >= seen) s[r / X::C][r % X::C] = -INFINITY;
            }
            // The largest of the lane's own scores says whether the column's has grown: only then do its lanes ask each other.
            float high = score(0);
#pragma unroll
            for (int r = 1; r < R; ++r) high = fmaxf(high, score(r));
            if (__any(high > limit)) {
                const float now = fmaxf(top, column_max<M>(high));
                const float less = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((top - now) * c);
                top = now;
                limit = now + grows;
                if ((limit - now) * c > GROWS) limit = now; // (rounded up, or past 32 bits' largest)
                far = __any(top != -INFINITY && !(fabsf(top * c) < FAR));
#pragma unroll
                for (int e = 0; e < 4; ++e) sums[e] *= less;
#pragma unroll
                for (int d = 0; d < DH / M; ++d) o[d] *= less;
            }
            // Where the largest, in powers of two, is FAR and more from zero, it is subtracted from the scores as they are: there the rounding of its product with the scale
            // is a factor that counts (2^4 at 1e8; f16 leaves room for 2).  Nearer, that is at most 1 + 2^-11, no more than the score's own rounding makes, and the subtraction is
            // spared (2 x 8192 causal rows: 537 us with it, 524 without).
            const float base = top == -INFINITY ? 0.f : top;
            if (far) {
#pragma unroll
                for (int r = 0; r < R; ++r) s[r / X::C][r % X::C] -= base;
            }
            const float about = far ? -LIFT : __builtin_fmaf(base, c, -LIFT);
            typename X::frag p[TK / X::KK];
            float chance[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                chance[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(score(r), c, -about));
                sums[r % 4] += chance[r];
            }
#pragma unroll
            for (int u = 0; u < TK / X::KK; ++u) p[u] = pack_eight<T>(chance + 8 * u);
#pragma unroll
            for (int u = 0; u < TK / X::KK; ++u)
#pragma unroll
                for (int d = 0; d < DH / M; ++d) {
                    o[d] = X::mul(L::template across<M>(across, u * X::KK, d * M, TK * L::PB), p[u], o[d]);
                    one_by_one<T>();
                }
            in_turn<T, TK / X::KK * (DH / M), 2, AHEAD>();
        }
    }
    const float sum = column_sum<M>(sums[0] + sums[1] + (sums[2] + sums[3]));
    row = row0 + again(col), pos = attn_position(a, row), head = at.kv * a.group + (row - pos * a.group);
    const float base = top == -INFINITY ? 0.f : top;
    if (split.count > 1) { // a part of a row: results, and their sum about the largest score
        const int64_t slot = attn_slot(a, at);
        if (g == 0 && half == 0) ((float2 *)a.part_sums)[slot * a.columns + row - at.part * a.columns] = make_float2(top != -INFINITY || sum != sum ? base : -INFINITY, sum);
        store_part<M, WAVES>(a.part, slot, wave, lane, 1.f, o);
        return;
    }
    const int64_t index = ((int64_t)at.n * a.heads + head) * a.Lq + pos;
    const float lse = seen ? attn_log_sum(base, a.scale, sum, LIFT) : -INFINITY;
    if (g == 0 && half == 0 && a.lse && row < rows) a.lse[index] = lse;
    const float inv = seen ? lse == lse ? 1.f / sum : lse : 0.f;
    if (row >= rows) return;
    T *const o_row = (T *)a.o + at.n * a.o_image + pos * a.o_row + head * a.o_head;
    auto result = [&](float sum) { return seen ? sum * inv : 0.f; }; // (a row that sees nothing: weights of zero, which times values that are not finite are not)
#pragma unroll
    for (int d = 0; d < DH / M; ++d)
#pragma unroll
        for (int r = 0; r < X::C; r += 4)
            store_four<T>(o_row, e0 + d * M + X::row_of(r, g), a.D, result(o[d][r]), result(o[d][r + 1]), result(o[d][r + 2]), result(o[d][r + 3]));
}

// ---------------------------------------------------------------- backward

// f16 numbers reach from 2^-24 to 2^16 only.  A column's numbers are multiplied by a power of two that brings the largest so far to 2^11 .. 2^12 before
// they are rounded; when one of 2^15 comes, what has been summed is scaled down with the factor, which that room makes rare (f16, 2 x 4096 causal rows of 16
// heads of 128: 543 us, brought to 2^14 558).  Probabilities of a key too: it may have little weight in all rows, whose gradients may be large.  (bf16 and f32 need none.)
template <typename T> struct Lift {
    static constexpr bool USED = std::is_same<T, f16_t>::value;
    float by = USED ? 0x1p100f : 1.f;
    __device__ __forceinline__ bool over(float high) const { return high * by > 0x1p15f; }
    // For numbers of a column whose largest magnitude is `high`; returns what to multiply the column's sums by.
    __device__ __forceinline__ float fit(float high)
    {
        if (!over(high)) return 1.f;
        const float now = __builtin_ldexpf(1.f, 11 + 127 - (int)(__float_as_uint(high) >> 23)), less = now / by;
        by = now;
        return less;
    }
    // The same of the lanes' own largest numbers; they ask each other only where one is over.
    template <int M, typename ACC, int COUNT> __device__ __forceinline__ void follow(float high, ACC (&sums)[COUNT])
    {
        if (!__any(over(high))) return;
        const float less = fit(column_max<M>(high));
#pragma unroll
        for (int d = 0; d < COUNT; ++d) sums[d] *= less;
    }
};

// Two wavefronts that have halves of the scores' and products' sums of two blocks: each finishes one (the second one's is the second), in `inbox` + wave * 2 KB,
// where the other one's half comes and where what it made of the block (with `make`: four scores and products to four numbers, and whatever else) stays for the
// other to read.
template <typename T, int M, typename L, typename ACC, typename F>
__device__ __forceinline__ f32x4 finish_block(bool second, const ACC (&s)[2], const ACC (&dp)[2], uint32_t inbox, int wave, F &&make)
{
    const uint32_t mine = inbox + wave * 2048, others = inbox + (wave ^ 1) * 2048;
    f32x4 score, product, give_s, give_p;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        score[e] = second ? s[1][e] : s[0][e], give_s[e] = second ? s[0][e] : s[1][e];
        product[e] = second ? dp[1][e] : dp[0][e], give_p[e] = second ? dp[0][e] : dp[1][e];
    }
    L::write(others, give_s);
    L::write(others + 1024, give_p);
    attn_barrier();
    score += L::template read<f32x4>(mine);
    product += L::template read<f32x4>(mine + 1024);
    f32x4 made;
#pragma unroll
    for (int e = 0; e < 4; ++e) made[e] = make(e, score[e], product[e]);
    L::write(mine, made);
    attn_barrier();
    return made;
}

// Columns: query rows, as above.  dq = scale sum over keys of dS k, dS = P (do v - delta), P = exp(score - lse).  Three products a tile; bound as forward.
template <typename T, int DP, int M, int WAVES, int SHARE, int TK, int NBUF> struct DqShape {
    static constexpr int LDS = NBUF * 2 * TK * Tile<T, DP>::PB + (SHARE > 1 ? WAVES * 2048 : 0);
};
template <typename T, int DP, int M, int WAVES, int SHARE, int TK, int NBUF> __device__ __forceinline__ void attention_dq(const AttnArgs &a, int block, uint8_t *lds)
{
    typedef Mma<T, M> X;
    typedef Tile<T, DP> L;
    constexpr int STEP = M > X::KK ? M : X::KK, BLOCKS = STEP / M, R = STEP / X::NG, DH = DP / SHARE, AHEAD = 6; // keys at a time, elements of a wavefront
    constexpr int TILES = NBUF * 2 * TK * L::PB, SWAP = 2048;
    static_assert(SHARE == 1 || (BLOCKS == SHARE && X::C == 4 && TK == STEP), "of two wavefronts each finishes the scores of one block, once a tile");
    AttnPlace at;
    if (!attn_place(a, block, &at)) return;
    if (a.causal) at.part = a.parts - 1 - at.part;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64), col = lane % M, g = lane / M;
    const int q_len = attn_length(a.q_len, at.n, a.Lq), k_len = attn_length(a.k_len, at.n, a.Lk), off = k_len - q_len;
    const int half = SHARE > 1 ? wave % SHARE : 0, e0 = half * DH; // which elements
    const int row0 = (at.part * (WAVES / SHARE) + wave / SHARE) * M, rows = a.Lq * a.group;
    const int row = row0 + col, pos = attn_position(a, row), head = at.kv * a.group + (row - pos * a.group);
    const bool here = row < rows, there = here && pos < q_len;
    const int seen = there ? (a.causal ? max(0, min(k_len, pos + off + 1)) : k_len) : 0;
    auto last_seen = [&](int last_row) { const int p = attn_position(a, min(last_row, rows - 1)); return a.causal ? max(0, min(k_len, min(p, q_len - 1) + off + 1)) : k_len; };
    const bool any = row0 < rows && attn_position(a, row0) < q_len;
    const int most = any ? last_seen(row0 + M - 1) : 0;
    const int least = row0 + M <= rows && attn_position(a, row0 + M - 1) < q_len ? (a.causal ? max(0, min(k_len, attn_position(a, row0) + off + 1)) : k_len) : 0;
    const AttnSplit split = attn_split(a, attn_key_tiles(a, q_len, k_len, at.part), at.split);
    if (at.split >= split.count) return;
    const int from = split.from, to = split.to;

    const uint8_t *const k = (const uint8_t *)a.k + (at.n * a.k_image + at.kv * a.k_head) * (int64_t)sizeof(T);
    const uint8_t *const v = (const uint8_t *)a.v + (at.n * a.v_image + at.kv * a.v_head) * (int64_t)sizeof(T);
    const int k_bytes = (int)a.k_row * (int)sizeof(T), v_bytes = (int)a.v_row * (int)sizeof(T);
    auto load = [&](int t) {
        uint8_t *const tile = lds + (t - from) % NBUF * (2 * TK * L::PB);
        const int first = t * TK;
        L::template load<TK, WAVES>(k + (int64_t)first * k_bytes, k_bytes, k_len - first, a.D, tile, tid, wave);
        L::template load<TK, WAVES>(v + (int64_t)first * v_bytes, v_bytes, k_len - first, a.D, tile + TK * L::PB, tid, wave);
    };
    if (from < to) load(from);

    typename X::frag q[DH / X::KK], dy[DH / X::KK];
    const T *const q_row = (const T *)a.q + at.n * a.q_image + pos * a.q_row + head * a.q_head;
    const T *const dy_row = (const T *)a.dy + at.n * a.o_image + pos * a.o_row + head * a.o_head;
#pragma unroll
    for (int s = 0; s < DH / X::KK; ++s) {
        q[s] = row_piece<T>(q_row, there, e0 + s * X::KK + 8 * g, a.D);
        dy[s] = row_piece<T>(dy_row, there, e0 + s * X::KK + 8 * g, a.D);
    }
    const int64_t index = ((int64_t)at.n * a.heads + head) * a.Lq + pos;
    const float less = there ? a.row_lse[index] * a.scale * kLog2E : -INFINITY, delta = there ? a.row_delta[index] : 0.f;

    wait_known_loads();
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_t)lds, mine = lds0 + e0 * (int)sizeof(T);
    const uint32_t along0 = mine + L::template along_at<M>(col, g), across0 = mine + L::template across_at<M>(lane);
    typename X::acc dq[DH / M] = {};
    Lift<T> lift;
    const float c = a.scale * kLog2E;
    for (int t = from; t < to; ++t) {
        wait_loads();
        attn_barrier();
        if (NBUF > 1 && t + 1 < to) load(t + 1);
        const uint32_t tile = (t - from) % NBUF * (2 * TK * L::PB), along = NBUF == 1 ? again(along0) : along0 + tile, across = NBUF == 1 ? again(across0) : across0 + tile;
#pragma unroll
        for (int h = 0; h < TK; h += STEP) {
            const int first = t * TK + h;
            if (SHARE == 1 && first >= most) break;
            typename X::acc s[BLOCKS], dp[BLOCKS];
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) s[b] = dp[b] = typename X::acc{};
#pragma unroll
            for (int i = 0; i < DH / X::KK; ++i)
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    s[b] = X::mul(L::template along<M>(along, i, (h + b * M) * L::PB), q[i], s[b]);
                    one_by_one<T>();
                    dp[b] = X::mul(L::template along<M>(along, i, (TK + h + b * M) * L::PB), dy[i], dp[b]);
                    one_by_one<T>();
                }
            in_turn<T, 2 * BLOCKS * (DH / X::KK), 1, AHEAD>();
            float ds[R], high = 0.f;
            if constexpr (SHARE == 1) {
#pragma unroll
                for (int r = 0; r < R; ++r) ds[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r / X::C][r % X::C], c, less)) * (dp[r / X::C][r % X::C] + delta);
                if (first + STEP > least) {
#pragma unroll
                    for (int r = 0; r < R; ++r) ds[r] = first + X::row_of(r, g) < seen ? ds[r] : 0.f;
                }
            } else {
                const bool second = half != 0;
                const f32x4 own = finish_block<T, M, L>(second, s, dp, lds0 + TILES + lane * 16, wave, [&](int e, float score, float product) {
                    const float z = __builtin_amdgcn_exp2f(__builtin_fmaf(score, c, less)) * (product + delta);
                    return first + (second ? M : 0) + X::row_of(e, g) < seen ? z : 0.f;
                });
                const f32x4 other = L::template read<f32x4>(lds0 + TILES + lane * 16 + (wave ^ 1) * SWAP);
#pragma unroll
                for (int e = 0; e < 4; ++e) ds[e] = second ? other[e] : own[e], ds[4 + e] = second ? own[e] : other[e];
            }
            if constexpr (Lift<T>::USED) {
#pragma unroll
                for (int r = 0; r < R; ++r) high = fmaxf(high, fabsf(ds[r]));
                lift.template follow<M>(high, dq);
            }
            typename X::frag p[STEP / X::KK];
#pragma unroll
            for (int r = 0; r < R; ++r) ds[r] = Lift<T>::USED ? ds[r] * lift.by : ds[r];
#pragma unroll
            for (int u = 0; u < STEP / X::KK; ++u) p[u] = pack_eight<T>(ds + 8 * u);
#pragma unroll
            for (int u = 0; u < STEP / X::KK; ++u)
#pragma unroll
                for (int d = 0; d < DH / M; ++d) {
                    dq[d] = X::mul(L::template across<M>(across, h + u * X::KK, d * M, 0), p[u], dq[d]);
                    one_by_one<T>();
                }
            in_turn<T, STEP / X::KK * (DH / M), 2, AHEAD>();
        }
        if (NBUF == 1 && t + 1 < to) {
            attn_barrier();
            load(t + 1);
        }
    }
    if (!seen) { // (as forward)
#pragma unroll
        for (int d = 0; d < DH / M; ++d) dq[d] = typename X::acc{};
    }
    const float by = a.scale / lift.by;
    if (split.count > 1) {
        store_part<M, WAVES>(a.part, attn_slot(a, at), wave, lane, by, dq);
        return;
    }
    if (!here) return;
    T *const out = (T *)a.dq + at.n * a.q_image + pos * a.q_row + head * a.q_head;
#pragma unroll
    for (int d = 0; d < DH / M; ++d)
#pragma unroll
        for (int r = 0; r < X::C; r += 4) store_four<T>(out, e0 + d * M + X::row_of(r, g), a.D, dq[d][r] * by, dq[d][r + 1] * by, dq[d][r + 2] * by, dq[d][r + 3] * by);
}

// Columns: key rows.  dv = sum over queries of P do, dk = scale sum of dS q, over all heads that share the keys.  DK, DV: which of the two (both where the
// registers hold both).  Of 128 elements of 16 bits the values lie in LDS: with them in registers there are none left for operands that are on their way
// (2 x 4096 causal rows of 16 heads, the whole call: 480 us, from LDS 471, with three reads for two products instead of two).  Bound: rows of 128 and less by the matrix pipe, with seven
// products in both halves (that call: 448 us in the kernel, 1.07 PFLOP/s); one head of 512 by the three barriers of a tile and LDS, which hold one workgroup to a compute unit (4 x 1024 rows: 63 us).
template <typename T, int DP, int M, int WAVES, int SHARE, int TQ, int NBUF, bool DK, bool DV> struct DkvShape {
    static constexpr bool FROM_LDS = DK && DV && sizeof(T) == 2 && DP == 128;
    static constexpr int LDS = NBUF * (2 * TQ * Tile<T, DP>::PB + 512) + (FROM_LDS ? WAVES * M * Tile<T, DP>::PB : 0) + (SHARE > 1 ? WAVES * 2048 : 0);
};
template <typename T, int DP, int M, int WAVES, int SHARE, int TQ, int NBUF, bool DK, bool DV> __device__ __forceinline__ void attention_dkv(const AttnArgs &a, int block, uint8_t *lds)
{
    typedef Mma<T, M> X;
    typedef Tile<T, DP> L;
    constexpr int STEP = M > X::KK ? M : X::KK, BLOCKS = STEP / M, R = STEP / X::NG, DH = DP / SHARE, AHEAD = 4;
    constexpr int BUF = 2 * TQ * L::PB + 512; // queries, gradients, 64 log-sums, 64 deltas
    constexpr bool FROM_LDS = DkvShape<T, DP, M, WAVES, SHARE, TQ, NBUF, DK, DV>::FROM_LDS;
    constexpr int TILES = NBUF * BUF + (FROM_LDS ? WAVES * M * L::PB : 0), SWAP = 2048;
    static_assert(TQ <= 64, "a wavefront loads a tile's log-sums at once");
    static_assert(SHARE == 1 || (BLOCKS == SHARE && X::C == 4 && TQ == STEP), "of two wavefronts each finishes the scores of one block, once a tile");
    AttnPlace at;
    if (!attn_place(a, block, &at)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64), col = lane % M, g = lane / M;
    const int q_len = attn_length(a.q_len, at.n, a.Lq), k_len = attn_length(a.k_len, at.n, a.Lk), off = k_len - q_len;
    const int half = SHARE > 1 ? wave % SHARE : 0, e0 = half * DH;
    const int key0 = (at.part * (WAVES / SHARE) + wave / SHARE) * M, key = key0 + col;
    const bool here = key < a.Lk, there = key < k_len;
    // all heads' queries one after the other
    int skip;
    const int each = attn_query_tiles(a, q_len, k_len, at.part, &skip);
    const AttnSplit split = attn_split(a, each * a.group, at.split);
    if (at.split >= split.count) return;
    const int from = split.from, to = split.to;

    const int q_bytes = (int)a.q_row * (int)sizeof(T), y_bytes = (int)a.o_row * (int)sizeof(T);
    struct Walk { // tile by tile, head by head
        int head, tile, buffer;
        __device__ __forceinline__ void next(int each)
        {
            const bool last = tile + 1 == each;
            head += last ? 1 : 0;
            tile = last ? 0 : tile + 1;
            buffer = NBUF - 1 - buffer;
        }
    };
    const int head0 = from ? from / each : 0;
    Walk now{head0, from - head0 * each, 0}, ahead = now;
    auto load = [&](const Walk &w) {
        uint8_t *const tile = lds + w.buffer * BUF;
        const int first = (skip + w.tile) * TQ, head = at.kv * a.group + w.head;
        const uint8_t *const q = (const uint8_t *)a.q + (at.n * a.q_image + head * a.q_head + (int64_t)first * a.q_row) * (int64_t)sizeof(T);
        const uint8_t *const y = (const uint8_t *)a.dy + (at.n * a.o_image + head * a.o_head + (int64_t)first * a.o_row) * (int64_t)sizeof(T);
        L::template load<TQ, WAVES>(q, q_bytes, q_len - first, a.D, tile, tid, wave);
        L::template load<TQ, WAVES>(y, y_bytes, q_len - first, a.D, tile + TQ * L::PB, tid, wave);
        const int64_t index = ((int64_t)at.n * a.heads + head) * a.Lq + first;
        if (wave == 0) {
            const int bytes = min(64, q_len - first) * 4;
            __amdgpu_buffer_rsrc_t l = __builtin_amdgcn_make_buffer_rsrc((void *)(a.row_lse + index), 0, bytes, 0x00020000);
            __amdgpu_buffer_rsrc_t d = __builtin_amdgcn_make_buffer_rsrc((void *)(a.row_delta + index), 0, bytes, 0x00020000);
            const uint32_t ones = again_scalar(~0u), off = __builtin_amdgcn_mbcnt_hi(ones, __builtin_amdgcn_mbcnt_lo(ones, 0)) * 4;
            load_to_lds4(l, off, tile + 2 * TQ * L::PB);
            load_to_lds4(d, off, tile + 2 * TQ * L::PB + 256);
        }
    };
    if (from < to) {
        load(ahead);
        if (FROM_LDS) {
            const int base = at.part * (WAVES / SHARE) * M;
            L::template load<WAVES * M, WAVES>((const uint8_t *)((const T *)a.v + at.n * a.v_image + at.kv * a.v_head + (int64_t)base * a.v_row), (int)a.v_row * (int)sizeof(T), k_len - base,
                                               a.D, lds + NBUF * BUF, tid, wave);
        }
    }

    typename X::frag k[DH / X::KK], v[DK && !FROM_LDS ? DH / X::KK : 1];
    const T *const k_row = (const T *)a.k + at.n * a.k_image + key * a.k_row + at.kv * a.k_head;
    const T *const v_row = (const T *)a.v + at.n * a.v_image + key * a.v_row + at.kv * a.v_head;
#pragma unroll
    for (int s = 0; s < DH / X::KK; ++s) {
        k[s] = row_piece<T>(k_row, there, e0 + s * X::KK + 8 * g, a.D);
        if constexpr (DK && !FROM_LDS) v[s] = row_piece<T>(v_row, there, e0 + s * X::KK + 8 * g, a.D);
    }

    wait_known_loads();
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_t)lds, mine = lds0 + e0 * (int)sizeof(T);
    const uint32_t along0 = mine + L::template along_at<M>(col, g), across0 = mine + L::template across_at<M>(lane);
    const uint32_t values = lds0 + NBUF * BUF + L::template along_at<M>(wave * M + col, g);
    typename X::acc dk[DK ? DH / M : 1] = {}, dv[DV ? DH / M : 1] = {};
    Lift<T> lift, lift_p; // of score gradients, of probabilities
    const float c = a.scale * kLog2E;
    for (int t = from; t < to; ++t) {
        wait_loads();
        attn_barrier();
        ahead.next(each);
        if (NBUF > 1 && t + 1 < to) load(ahead);
        // queries; gradients behind them (where they lie in one place tile after tile, their addresses are computed anew all the same: kept, they take the registers)
        const uint32_t tile = now.buffer * BUF, along = NBUF == 1 ? again(along0) : along0 + tile, across = NBUF == 1 ? again(across0) : across0 + tile, sums = lds0 + tile + 2 * TQ * L::PB + 16 * g;
        const int pos0 = (skip + now.tile) * TQ;
        now.next(each);
#pragma unroll
        for (int h = 0; h < TQ; h += STEP) {
            if (SHARE == 1 && pos0 + h >= q_len) break;
            const int behind = a.causal ? key0 - off - (pos0 + h) : 0; // query row r of these sees the wavefront's keys 0 .. r - behind
            if (SHARE == 1 && behind >= STEP) continue;
            // The sums begin with what is subtracted from them: minus delta, and minus lse / scale (f32: that one afterwards, for its 24 bits' sake).
            constexpr bool AFTER = sizeof(T) == 4 || SHARE > 1;
            auto row_sums = [&](int r, int which) { return L::template read<f32x4>(sums + which * 256 + (h + X::row_of(r, 0)) * 4); };
            typename X::acc s[BLOCKS], dp[BLOCKS];
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                s[b] = dp[b] = typename X::acc{};
#pragma unroll
                for (int r = 0; r < X::C; r += 4) {
                    const f32x4 less = AFTER ? f32x4{} : row_sums(b * X::C + r, 0), mean = SHARE > 1 ? f32x4{} : row_sums(b * X::C + r, 1);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[b][r + e] = less[e], dp[b][r + e] = mean[e];
                }
            }
#pragma unroll
            for (int i = 0; i < DH / X::KK; ++i)
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    s[b] = X::mul(L::template along<M>(along, i, (h + b * M) * L::PB), k[i], s[b]);
                    one_by_one<T>();
                    if constexpr (DK) {
                        typename X::frag value;
                        if constexpr (FROM_LDS) value = L::template along<M>(values, i, 0);
                        else value = v[i];
                        dp[b] = X::mul(L::template along<M>(along, i, (TQ + h + b * M) * L::PB), value, dp[b]);
                        one_by_one<T>();
                    }
                }
            in_turn<T, BLOCKS * (DH / X::KK), FROM_LDS ? 3 : 2, AHEAD / 2, SHARE == 1 ? R / 2 : 0, 2>();
            float pr[R], ds[R];
            if constexpr (SHARE == 1) {
#pragma unroll
                for (int r = 0; r < R; r += 4) {
                    const f32x4 less = AFTER ? row_sums(r, 0) : f32x4{};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float score = s[(r + e) / X::C][(r + e) % X::C];
                        pr[r + e] = __builtin_amdgcn_exp2f(AFTER ? __builtin_fmaf(score, c, less[e] * c) : score * c);
                        ds[r + e] = DK ? pr[r + e] * dp[(r + e) / X::C][(r + e) % X::C] : 0.f;
                    }
                }
                if (behind > 1 - M && a.causal) {
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        if (X::row_of(r, g) - behind < col) pr[r] = ds[r] = 0.f;
                }
            } else {
                const bool second = half != 0;
                const uint32_t swap = lds0 + TILES + lane * 16, block = sums + (h + (second ? M : 0)) * 4;
                const f32x4 less = L::template read<f32x4>(block), mean = L::template read<f32x4>(block + 256);
                f32x4 chance;
                const f32x4 own = finish_block<T, M, L>(second, s, dp, swap, wave, [&](int e, float score, float product) {
                    float p = __builtin_amdgcn_exp2f(__builtin_fmaf(score, c, less[e] * c)), z = p * (product + mean[e]);
                    if (a.causal && X::row_of(e, g) + (second ? M : 0) - behind < col) p = z = 0.f;
                    chance[e] = p;
                    if (e == 3) L::write(swap + wave * SWAP + 1024, chance);
                    return z;
                });
                const f32x4 other = L::template read<f32x4>(swap + (wave ^ 1) * SWAP), other_chance = L::template read<f32x4>(swap + (wave ^ 1) * SWAP + 1024);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    ds[e] = second ? other[e] : own[e], ds[4 + e] = second ? own[e] : other[e];
                    pr[e] = second ? other_chance[e] : chance[e], pr[4 + e] = second ? chance[e] : other_chance[e];
                }
            }
            if constexpr (Lift<T>::USED && DK) {
                float high = 0.f;
#pragma unroll
                for (int r = 0; r < R; ++r) high = fmaxf(high, fabsf(ds[r]));
                lift.template follow<M>(high, dk);
            }
            if constexpr (Lift<T>::USED && DV) {
                float high = 0.f;
#pragma unroll
                for (int r = 0; r < R; ++r) high = fmaxf(high, pr[r]);
                lift_p.template follow<M>(high, dv);
            }
            typename X::frag p[STEP / X::KK], z[STEP / X::KK];
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (Lift<T>::USED) pr[r] *= lift_p.by, ds[r] *= lift.by;
#pragma unroll
            for (int u = 0; u < STEP / X::KK; ++u) p[u] = pack_eight<T>(pr + 8 * u), z[u] = pack_eight<T>(ds + 8 * u);
#pragma unroll
            for (int u = 0; u < STEP / X::KK; ++u)
#pragma unroll
                for (int d = 0; d < DH / M; ++d) {
                    if constexpr (DV) dv[d] = X::mul(L::template across<M>(across, h + u * X::KK, d * M, TQ * L::PB), p[u], dv[d]);
                    if constexpr (DK) dk[d] = X::mul(L::template across<M>(across, h + u * X::KK, d * M, 0), z[u], dk[d]);
                    one_by_one<T>();
                }
            in_turn<T, 2 * (STEP / X::KK) * (DH / M), 2, AHEAD>();
        }
        if (NBUF == 1 && t + 1 < to) {
            attn_barrier();
            load(ahead);
        }
    }
    const float by_k = a.scale / lift.by, by_v = 1.f / lift_p.by;
    auto write = [&](const auto &sums, float by, T *out) {
#pragma unroll
        for (int d = 0; d < DH / M; ++d)
#pragma unroll
            for (int r = 0; r < X::C; r += 4) {
                const float w[4] = {there ? sums[d][r] * by : 0.f, there ? sums[d][r + 1] * by : 0.f, there ? sums[d][r + 2] * by : 0.f, there ? sums[d][r + 3] * by : 0.f};
                store_four<T>(out, e0 + d * M + X::row_of(r, g), a.D, w[0], w[1], w[2], w[3]);
            }
    };
    if (split.count > 1) {
        const int64_t slot = attn_slot(a, at);
        if constexpr (DK)
            if (a.dk) store_part<M, WAVES>(a.part_k, slot, wave, lane, by_k, dk);
        if constexpr (DV)
            if (a.dv) store_part<M, WAVES>(a.part_v, slot, wave, lane, by_v, dv);
        return;
    }
    if (!here) return;
    if constexpr (DK)
        if (a.dk) write(dk, by_k, (T *)a.dk + at.n * a.k_image + key * a.k_row + at.kv * a.k_head);
    if constexpr (DV)
        if (a.dv) write(dv, by_v, (T *)a.dv + at.n * a.v_image + key * a.v_row + at.kv * a.v_head);
}

// Both in one launch: the first `split` workgroups do keys' gradients, which take longer, the others queries'.  What is short then fills the compute units that the
// long leave, and a small launch's beginning and end are passed once.
template <typename T, int DP, bool DK, bool DV>
__global__ __launch_bounds__(attn_shape(sizeof(T), DP, ATTN_DQ).waves * 64, 2) void attention_backward_kernel(AttnArgs by_q, AttnArgs by_k, int split)
{
    constexpr AttnShape q = attn_shape(sizeof(T), DP, ATTN_DQ), k = attn_shape(sizeof(T), DP, ATTN_DKV);
    static_assert(q.waves == k.waves, "one launch");
    typedef DqShape<T, DP, q.m, q.waves, q.share, q.tile, q.buffers> Dq;
    typedef DkvShape<T, DP, k.m, k.waves, k.share, k.tile, k.buffers, DK, DV> Dkv;
    __shared__ alignas(256) uint8_t lds[Dq::LDS > Dkv::LDS ? Dq::LDS : Dkv::LDS];
    if ((int)blockIdx.x < split) attention_dkv<T, DP, k.m, k.waves, k.share, k.tile, k.buffers, DK, DV>(by_k, blockIdx.x, lds);
    else if constexpr (DK) attention_dq<T, DP, q.m, q.waves, q.share, q.tile, q.buffers>(by_q, blockIdx.x - split, lds); // (dv alone: no launch for queries)
}

// ---------------------------------------------------------------- launches

// Workgroups of a launch's cut, in eights (attn_place).
inline uint32_t attn_blocks(const AttnArgs &a) { return (uint32_t)(((int64_t)a.N * a.kv_heads * a.parts * a.splits + 7) / 8 * 8); }

template <typename T, int DP> hipError_t attention_forward_width(int kind, const AttnArgs &a, hipStream_t s)
{
    const auto launch = [&](auto few) {
        constexpr AttnShape h = attn_shape(sizeof(T), DP, decltype(few)::value);
        hipLaunchKernelGGL((attention_kernel<T, DP, h.m, h.waves, h.share, h.tile, h.buffers, h.occupancy>), dim3(attn_blocks(a)), dim3(h.waves * 64), 0, s, a);
    };
    kind == ATTN_FEW ? launch(std::integral_constant<int, ATTN_FEW>()) : launch(std::integral_constant<int, ATTN_FORWARD>());
    return hipGetLastError();
}

template <typename T, int DP> hipError_t attention_backward_width(const AttnArgs &by_q, const AttnArgs &by_k, hipStream_t s)
{
    const dim3 threads(attn_shape(sizeof(T), DP, ATTN_DQ).waves * 64);
    const auto launch = [&](auto dk, auto dv, bool keys, bool queries) {
        const uint32_t first = keys ? attn_blocks(by_k) : 0, blocks = first + (queries ? attn_blocks(by_q) : 0);
        if (blocks) hipLaunchKernelGGL((attention_backward_kernel<T, DP, decltype(dk)::value, decltype(dv)::value>), dim3(blocks), threads, 0, s, by_q, by_k, (int)first);
    };
    if constexpr (attn_dk_dv_at_once(sizeof(T), DP)) {
        launch(std::true_type(), std::true_type(), by_k.dk || by_k.dv, by_q.dq);
    } else {
        if (by_k.dk || by_q.dq) launch(std::true_type(), std::false_type(), by_k.dk, by_q.dq);
        if (by_k.dv) launch(std::false_type(), std::true_type(), true, false);
    }
    return hipGetLastError();
}

// Calls f with the width of a kernel for rows of D elements.
template <typename T, typename F> hipError_t attention_with_width(int D, F &&f)
{
    switch (attn_width(sizeof(T), D)) {
    case 32: return f(std::integral_constant<int, 32>());
    case 64: return f(std::integral_constant<int, 64>());
    case 96: return f(std::integral_constant<int, 96>());
    case 128: return f(std::integral_constant<int, 128>());
    case 192: return f(std::integral_constant<int, sizeof(T) == 2 ? 192 : 256>());
    case 256: return f(std::integral_constant<int, 256>());
    default: return f(std::integral_constant<int, 512>());
    }
}
template <typename T> hipError_t attention_forward(int kind, const AttnArgs &a, hipStream_t s)
{
    return attention_with_width<T>(a.D, [&](auto width) { return attention_forward_width<T, decltype(width)::value>(kind, a, s); });
}
template <typename T> hipError_t attention_backward(const AttnArgs &by_q, const AttnArgs &by_k, hipStream_t s)
{
    return attention_with_width<T>(by_q.D, [&](auto width) { return attention_backward_width<T, decltype(width)::value>(by_q, by_k, s); });
}

} // namespace qrm
