// Softmax cross entropy of rows x_t against classes w_v, forward and backward,
// without storing the logits z_tv = scale <x_t, w_v>:
//
//   lse_t  = log sum_v exp z_tv
//   loss_t = lse_t - z_t,target + z_weight lse_t^2            (0 where ignored)
//   dz_tv  = g_t ((1 + 2 z_weight lse_t) p_tv - [v = target]), p = exp(z - lse)
//   dx     = scale dz w,   dw = scale dz^T x
//
// Four products of rows x classes x dim: z in the forward pass, z again in the
// backward pass (by pieces, turned into dz in registers), dz w and dz^T x. All
// run on the same matrix-core tiles of 16-bit operands (product()); what differs
// is how each operand lies in memory and what becomes of the result.
//
// float32 operands are cut into three bfloat16 planes of 8 significant bits
// each (exact: a = a0 + a1 + a2), and the product sums the six plane products
// that reach 24 bits: a0 b0, a0 b1, a1 b0, a0 b2, a2 b0, a1 b1. Each plane is what is
// left rounded to nearest, |a1| <= 2^-8 |a| and |a2| <= 2^-17 |a|, so that the rest is
// at most 2^-24 of a term, as a rounding is, and of either sign (truncated planes
// leave out up to 2^-21 and always towards 0, 2^-24.7 in the mean). bfloat16 matrix instructions run at 16 times the rate
// of float32 ones, so six of them cost 3/8 of one float32 product.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "apml_internal.h"
#include "device_common.h"
#include "linear_ce.h"

namespace apml {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));

using lds_char = __attribute__((address_space(3))) char;

// The rows' targets as the caller holds them.
constexpr int kIgnored = -1, kOutside = -2;
struct Targets {
    const void *at;
    bool is32;
    int classes;
    int64_t ignore;
    __device__ __forceinline__ int operator[](int64_t i) const
    {
        const int64_t t = is32 ? (int64_t)((const int32_t *)at)[i] : ((const int64_t *)at)[i];
        return t == ignore ? kIgnored : t < 0 || t >= classes ? kOutside : (int)t;
    }
};

// ---------------------------------------------------------------------------
// 16-bit elements
// ---------------------------------------------------------------------------

struct Bf16 {
    static constexpr float kUnit = 1.0f; // what 1 becomes in the stored gradient of the logits
    static __device__ __forceinline__ uint16_t from(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
    static __device__ __forceinline__ float to(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
    static __device__ __forceinline__ f32x4 mma(i16x8 a, i16x8 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    }
};

struct F16 {
    // Probabilities of many classes fall below half precision's range (2^-24 is
    // its smallest step): with the values between -1 and 1 stored times 2^14,
    // that step is 2^-38.
    static constexpr float kUnit = 16384.0f;
    static __device__ __forceinline__ uint16_t from(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
    static __device__ __forceinline__ float to(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
    static __device__ __forceinline__ f32x4 mma(i16x8 a, i16x8 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
    }
};

// float32 as it is, two 16-bit elements a value: a fragment's 16 bytes are four
// neighbours, one for each of four instructions, on either side alike.
struct F32 {
    static __device__ __forceinline__ f32x4 mma(i16x8 a, i16x8 b, f32x4 c)
    {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
        return c;
    }
};

// v cut into three bfloat16 values of 8 significant bits, each the nearest to what
// the ones before it leave: v = a + b + c exactly. ANY: also for values that round
// to infinity (beyond 2^128 - 2^119; their first plane is truncated), which the
// gradient of the logits, in units of the largest upstream gradient, does not have.
struct Planes {
    i16x8 a, b, c;
};
template <bool ANY> __device__ __forceinline__ Planes planes_of(const float (&v)[8])
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    i32x4 p[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) { // one conversion instruction a pair
        f32x2 left = {v[2 * i], v[2 * i + 1]};
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            uint32_t w = __builtin_bit_cast(uint32_t, __builtin_convertvector(left, bf16x2));
            if (ANY && k == 0) {
                if ((w & 0x7fffu) == 0x7f80u)
                    w = (w & 0xffff0000u) | __builtin_bit_cast(uint32_t, v[2 * i]) >> 16;
                if ((w & 0x7fff0000u) == 0x7f800000u)
                    w = (w & 0xffffu) | (__builtin_bit_cast(uint32_t, v[2 * i + 1]) & 0xffff0000u);
            }
            p[k][i] = (int)w;
            left = left - f32x2{__builtin_bit_cast(float, w << 16), __builtin_bit_cast(float, w & 0xffff0000u)};
        }
    }
    return {__builtin_bit_cast(i16x8, p[0]), __builtin_bit_cast(i16x8, p[1]), __builtin_bit_cast(i16x8, p[2])};
}

// The plane products of a float32 product.
constexpr int kPlaneProducts = 6;

// ---------------------------------------------------------------------------
// the product C[q][p] = sum_k P[p][k] Q[q][k]
// ---------------------------------------------------------------------------

// One operand: `rows` rows (the p or q axis) by `k` summed elements, either
// with k contiguous (row r, element k at r * ld + k) or with the rows
// contiguous (at k * ld + r). Rows beyond `rows` are read as the last one; the
// results they give are not stored. ld is a multiple of 8 and the base 16-byte
// aligned.
struct Operand {
    const uint16_t *base;
    int64_t sample; // elements from one sample to the next
    int64_t plane;  // and from one plane to the next
    int64_t ld;
    int rows;
    int k;          // elements of the summed axis that may be read
};

struct Product {
    Operand p, q;
    int steps;       // steps of kCeStep along the summed axis
    int tiles_p, tiles_q, samples, splits;
    int group;       // q tiles that a run of workgroups stays within
};

// Chunks that row k of a tile with ROWS columns is moved by: a transposing read
// takes 2 chunks each of k = 8 a .. 8 a + 3 for a = 0 .. 3, which then cover all
// banks twice (128 columns or more fill them with one row, 64 with two).
template <int ROWS> __device__ __forceinline__ int k_swizzle(int k)
{
    return ROWS >= 128 ? ((k & 3) | ((k >> 1) & 4)) << 1 : (((k >> 1) & 1) | ((k >> 2) & 2)) << 1;
}

// Byte offset, from the operand's base of a step, of what lane `lane` of load
// `j` (1 KB of the tile) fetches. With k contiguous the tile holds ROWS rows of
// 8 chunks of 16 bytes, chunk c of row r in slot c ^ (r & 7): the 16 rows that a
// fragment read touches then lie in different banks (EIGHTS: the rows that
// such a fragment touches). With the rows contiguous it holds kCeStep rows of ROWS / 8
// chunks, moved by k_swizzle for the same reason (a transposing read touches the
// same columns of 16 rows).
// The base is that of row first_row (a tile of the padded rows may begin behind
// the last one).
template <bool KS> __device__ __forceinline__ int first_row(const Operand &o, int r0)
{
    return min(r0, KS ? (o.rows - 1) & ~7 : o.rows - 1);
}
template <bool EIGHTS> __device__ __forceinline__ int row_swizzle(int r) { return EIGHTS ? (r & 3) | ((r >> 1) & 4) : r & 7; }
template <int ROWS, bool KS, bool EIGHTS>
__device__ __forceinline__ uint32_t tile_offset(const Operand &o, int r0, int j, int lane, int k_left)
{
    if constexpr (!KS) {
        const int r = j * 8 + (lane >> 3);
        const int c = (lane & 7) ^ row_swizzle<EIGHTS>(r);
        const int row = min(r0 + r, o.rows - 1);
        return (uint32_t)((row - first_row<KS>(o, r0)) * o.ld + min(c, (k_left - 1) >> 3) * 8) * 2u;
    } else {
        constexpr int CH = ROWS / 8;
        const int k = j * (64 / CH) + lane / CH;
        const int c = (lane % CH) ^ k_swizzle<ROWS>(k);
        const int col = min(r0 + c * 8, (o.rows - 1) & ~7);
        return (uint32_t)(min(k, k_left - 1) * o.ld + (col - first_row<KS>(o, r0))) * 2u;
    }
}

// The same for an operand of float32 values (ld and base in 16-bit elements), of
// 16 chunks a row with k contiguous, else ROWS / 4 chunks: chunk c of row r in slot
// c ^ (r & 15), or of k in c ^ 4 (k / 8 & 3).
template <bool KS> __device__ __forceinline__ int float_swizzle(int r) { return KS ? (r >> 1) & 12 : r & 15; }
template <int ROWS, bool KS> __device__ __forceinline__ uint32_t float_offset(const Operand &o, int r0, int j, int lane, int k_left)
{
    constexpr int CH = KS ? ROWS / 4 : 16;
    const int r = j * (64 / CH) + lane / CH, c = (lane % CH) ^ float_swizzle<KS>(r);
    if constexpr (!KS) {
        const int row = min(r0 + r, o.rows - 1);
        return (uint32_t)((row - first_row<KS>(o, r0)) * o.ld) * 2u + min(c, (k_left - 1) >> 2) * 16u;
    } else {
        const int col = min(r0 + c * 4, (o.rows - 1) & ~3);
        return (uint32_t)(min(r, k_left - 1) * o.ld) * 2u + (col - first_row<KS>(o, r0)) * 4u;
    }
}

template <class T> using lds_ptr = __attribute__((address_space(3))) T *;

// Orders a wave's own accesses to shared memory.
__device__ __forceinline__ void wave_lds()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// Loads 16 bytes a lane straight into shared memory at lds + 16 lane. The
// caller waits for it (s_waitcnt vmcnt) before the barrier that hands the tile
// over; the compiler does not see it.
__device__ __forceinline__ void load_to_lds(i32x4 rsrc, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset),
                 "s"(rsrc)
                 : "memory");
}

__device__ __forceinline__ i32x4 buffer_at(uint64_t base)
{
    i32x4 r;
    r.x = (int)(uint32_t)base;
    r.y = (int)(uint32_t)(base >> 32) & 0xffff;
    r.z = -1; // the offsets stay in the operand by tile_offset
    r.w = 0x00020000;
    return r;
}

template <int N> __device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds_and_meet()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// The 16 x 32 fragment of a tile at rows r .. r + 15 and elements 32 h ..:
// lane l holds row l & 15, elements 8 (l >> 4) .. + 7. EIGHTS: fragment `i` of
// 32 rows holds rows 8 a + 4 (i & 1) .. + 3 for a = 0 .. 3, so that in the
// results a lane's values of two neighbouring fragments are 8 neighbours.
template <int ROWS, bool KS, bool EIGHTS>
__device__ __forceinline__ i16x8 fragment(const lds_char *tile, int r0, int i, int h, int lane)
{
    if constexpr (!KS) {
        const int row = EIGHTS ? r0 + (i >> 1) * 32 + ((lane & 12) << 1) + (i & 1) * 4 + (lane & 3) : r0 + i * 16 + (lane & 15);
        const int slot = (h * 4 + (lane >> 4)) ^ row_swizzle<EIGHTS>(row);
        return *(const __attribute__((address_space(3))) i16x8 *)(tile + row * 128 + slot * 16);
    } else {
        const int r = r0 + i * 16;
        // a transposing read gives lane i of 16 the column i of 4 rows of 16
        const int k = h * 32 + (lane >> 4) * 8 + ((lane & 15) >> 2);
        const int col = r + (lane & 3) * 4;
        const lds_char *at = tile + k * (ROWS * 2) + (((col >> 3) ^ k_swizzle<ROWS>(k)) << 4) + ((col & 7) << 1);
        using v4 = __attribute__((address_space(3))) i16x4;
        const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((v4 *)at);
        const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((v4 *)(at + 4 * ROWS * 2));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
}

// The three planes of such a fragment of float32 values.
template <int ROWS, bool KS>
__device__ __forceinline__ void float_fragment(const lds_char *tile, int r0, int i, int h, int lane, i16x8 (&planes)[3])
{
    const int r = r0 + i * 16 + (lane & 15), k = h * 32 + (lane >> 4) * 8;
    float v[8];
    if constexpr (!KS) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const f32x4 x = *(const __attribute__((address_space(3))) f32x4 *)(tile + r * 256 +
                                                                                (((k >> 2) + c) ^ float_swizzle<KS>(r)) * 16);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                v[c * 4 + u] = x[u];
        }
    } else {
        const lds_char *at = tile + k * (ROWS * 4) + (((r >> 2) ^ float_swizzle<KS>(k)) << 4) + ((r & 3) << 2);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            v[u] = *(const __attribute__((address_space(3))) float *)(at + u * (ROWS * 4));
    }
    const Planes x = planes_of<false>(v);
    planes[0] = x.a;
    planes[1] = x.b;
    planes[2] = x.c;
}

// The tile shapes. A workgroup takes TP x TQ results, its waves WP x WQ of them,
// with BUFS steps' tiles in shared memory. WOVEN: the fragments of the next half
// step are read between the matrix instructions of this one. TRIPLE, for float32: a
// step's tile holds all three planes of P and Q as it is, which is cut into planes
// on its way to the matrix cores, and gives all six products.
template <int TP_, int TQ_, int WP_, int WQ_, int BUFS_, bool WOVEN_ = false, bool TRIPLE_ = false> struct Shape {
    static constexpr int TP = TP_, TQ = TQ_, WP = WP_, WQ = WQ_, BUFS = BUFS_;
    static constexpr bool WOVEN = WOVEN_, TRIPLE = TRIPLE_;
    static_assert(!WOVEN || BUFS == 2, "two tiles in turn");
    static constexpr int waves = WP * WQ, threads = 64 * waves;
    static constexpr int SP = TP / WP / 16, SQ = TQ / WQ / 16; // 16 x 16 results of a wave
    static constexpr int at_q = TP * 128 * (TRIPLE ? 3 : 1); // bytes of P, then of Q
    static constexpr int stage = at_q + TQ * 128 * (TRIPLE ? 2 : 1);
    static constexpr int lds = stage * BUFS;
    static constexpr int LP = TP / 8 / waves;                                    // loads of a wave for P
    static constexpr int KQ = TQ / 8 * (TRIPLE ? 2 : 1);                         // KB of Q
    static constexpr int LQ = (KQ + waves - 1) / waves;                          // and for Q
};

struct Place {
    int p0, q0, sample, split; // where a workgroup's tile starts
    int wp, wq, lane;          // wave within the workgroup
    lds_char *lds;             // the wave's part of the tiles' memory, free once all waves are done with them
};

// ELEM: the elements; PLANES: float32 operands in three planes; PK, QK: the
// operand's rows are contiguous; Finish: what becomes of the results.
//
// Tiles go from memory to shared memory without passing registers, one step
// ahead (one and a half in the woven tile, three in that of 16 rows); the matrix cores take them as 16 x 32 fragments. P's rows come out along
// a lane's registers, Q's along the lanes: classes (or features) are P, so that
// the softmax's sums run mostly within a lane and results leave as neighbours.
// The large tile needs 64 KB of loads for 2048 cycles of matrix instructions a
// step, and keeps the matrix cores 60 to 65% busy at 2.0 to 2.25 GHz (power sets
// the clock): 1.28 to 1.43 PFLOP/s at 8192 x 131072 x 4096 and its gradients.
template <class ELEM, bool PLANES, bool PK, bool QK, class S, class Finish>
__device__ __forceinline__ void product(const Product &a, const Finish &finish, int block, int blocks)
{
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int lane = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    Place at;
    at.lane = lane;
    at.wp = wave % S::WP;
    at.wq = wave / S::WP;
    at.lds = (lds_char *)smem + wave * (S::lds / S::waves);
    {
        // The workgroups of an XCD take a run of tiles; within it, `group` q
        // tiles for one p tile after the other, so that the tiles in flight
        // share rows of both operands in that XCD's L2.
        int id = xcd_contiguous(block, blocks);
        const int per = a.tiles_p * a.tiles_q;
        at.split = id % a.splits;
        id /= a.splits;
        at.sample = id / per;
        id -= at.sample * per;
        const int g0 = id / (a.group * a.tiles_p) * a.group;
        const int gn = min(a.group, a.tiles_q - g0);
        id -= g0 * a.tiles_p;
        at.p0 = id / gn * S::TP;
        at.q0 = (g0 + id % gn) * S::TQ;
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char *)smem;
    // steps of this part of the sum
    const int first = (int)((int64_t)a.steps * at.split / a.splits);
    const int last = (int)((int64_t)a.steps * (at.split + 1) / a.splits);
    const int n = last - first, total = PLANES && !S::TRIPLE ? n * kPlaneProducts : n;

    uint32_t op[S::LP], oq[S::LQ];
    const auto offsets = [&](int step) {
        const int kp = min(kCeStep, a.p.k - step * kCeStep), kq = min(kCeStep, a.q.k - step * kCeStep);
#pragma unroll
        for (int j = 0; j < S::LP; ++j)
            op[j] = tile_offset<S::TP, PK, !PK>(a.p, at.p0, wave * S::LP + j, lane, kp);
#pragma unroll
        for (int j = 0; j < S::LQ; ++j)
            if constexpr (S::TRIPLE)
                oq[j] = float_offset<S::TQ, QK>(a.q, at.q0, (wave * S::LQ + j) % S::KQ, lane, kq);
            else
                oq[j] = tile_offset<S::TQ, QK, false>(a.q, at.q0, (wave * S::LQ + j) % S::KQ, lane, kq);
    };
    constexpr int size_q = S::TRIPLE ? 2 : 1; // in 16-bit elements
    const int64_t step_p = PK ? kCeStep * a.p.ld : kCeStep, step_q = QK ? kCeStep * a.q.ld : kCeStep * size_q;
    const uint64_t base_p = (uint64_t)(a.p.base + at.sample * a.p.sample + first_row<PK>(a.p, at.p0) * (PK ? 1 : a.p.ld));
    const uint64_t base_q = (uint64_t)(a.q.base + at.sample * a.q.sample + first_row<QK>(a.q, at.q0) * (QK ? size_q : a.q.ld));
    // A step that ends beyond an operand's summed axis clamps its offsets.
    const int ragged = (a.p.k < a.steps * kCeStep || a.q.k < a.steps * kCeStep) ? a.steps - 1 : -1;
    offsets(0);
    const auto load = [&](int i) {
        int step = first + i, pp = 0, pq = 0;
        if constexpr (PLANES && !S::TRIPLE) {
            const int prod = i / n;
            step = first + i - prod * n;
            pp = (0x120100 >> (4 * prod)) & 15; // planes 0 0 1 0 2 1
            pq = (0x102010 >> (4 * prod)) & 15; // planes 0 1 0 2 0 1
        }
        if (ragged >= 0 && (step == ragged || step == first))
            offsets(step);
        const uint32_t to = lds0 + (i % S::BUFS) * S::stage;
#pragma unroll
        for (int plane = 0; plane < (S::TRIPLE ? 3 : 1); ++plane) {
            const i32x4 rp = buffer_at(base_p + 2 * (uint64_t)(step * step_p + (pp + plane) * a.p.plane));
#pragma unroll
            for (int j = 0; j < S::LP; ++j)
                load_to_lds(rp, op[j], to + plane * (S::TP * 128) + (wave * S::LP + j) * 1024);
        }
        const i32x4 rq = buffer_at(base_q + 2 * (uint64_t)(step * step_q + pq * a.q.plane));
#pragma unroll
        for (int j = 0; j < S::LQ; ++j)
            load_to_lds(rq, oq[j], to + S::at_q + ((wave * S::LQ + j) % S::KQ) * 1024);
    };

    // what the finish needs of its rows is on its way during the products
    typename Finish::template Rows<S> rows;
    finish.fetch(a, at, rows);

    f32x4 acc[S::SP][S::SQ];
#pragma unroll
    for (int i = 0; i < S::SP; ++i)
#pragma unroll
        for (int j = 0; j < S::SQ; ++j)
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const auto read_p = [&](const lds_char *tp, int h, i16x8 (&fp)[S::SP]) {
#pragma unroll
        for (int k = 0; k < S::SP; ++k)
            fp[k] = fragment<S::TP, PK, !PK>(tp, at.wp * (S::SP * 16), k, h, lane);
    };
    const auto read = [&](int i, int h, i16x8 (&fp)[S::SP], i16x8 (&fq)[S::SQ]) {
        const lds_char *tp = (const lds_char *)smem + (i % S::BUFS) * S::stage;
#pragma unroll
        for (int j = 0; j < S::SQ; ++j)
            fq[j] = fragment<S::TQ, QK, false>(tp + S::at_q, at.wq * (S::SQ * 16), j, h, lane);
        read_p(tp, h, fp);
    };
    const auto multiply = [&](const i16x8 (&fp)[S::SP], const i16x8 (&fq)[S::SQ]) {
#pragma unroll
        for (int k = 0; k < S::SP; ++k)
#pragma unroll
            for (int j = 0; j < S::SQ; ++j)
                acc[k][j] = ELEM::mma(fp[k], fq[j], acc[k][j]);
    };

    // Every barrier says two things: a step's tile has arrived (each wave has
    // waited for its own loads), and every wave has read the tile whose place the
    // next loads take.
    if constexpr (S::WOVEN) {
        // With one workgroup a compute unit, its two waves a SIMD meet at every
        // barrier, and fragments read right after it leave the matrix cores idle
        // in both. So a half step's fragments are read one half step ahead, a read
        // after every one or two matrix instructions, and the barrier stands in
        // the middle of a step, with a half step's instructions ready behind it
        // (8192 x 131072 x 4096: 1.30 -> 1.43 PFLOP/s; with the reads ahead but
        // not woven in 1.39).
        constexpr int reads = S::SP * (PK ? 2 : 1) + S::SQ * (QK ? 2 : 1), products = S::SP * S::SQ;
        const auto weave = [] {
#pragma unroll
            for (int r = 0; r < reads; ++r) {
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0); // a read from shared memory
                __builtin_amdgcn_sched_group_barrier(0x008, products / reads, 0); // matrix instructions
            }
            __builtin_amdgcn_sched_group_barrier(0x008, products, 0);
        };
        static_assert(products >= reads, "");
        if (total > 0) {
            load(0);
            if (total > 1) {
                load(1);
                wait_loads<S::LP + S::LQ>();
            } else {
                wait_loads<0>();
            }
            wait_lds_and_meet();
            i16x8 p0[S::SP], q0[S::SQ], p1[S::SP], q1[S::SQ];
            read(0, 0, p0, q0);
            for (int i = 0; i < total; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                read(i, 1, p1, q1);
                multiply(p0, q0);
                weave();
                __builtin_amdgcn_sched_barrier(0);
                wait_loads<0>();
                wait_lds_and_meet();
                if (i + 2 < total)
                    load(i + 2);
                __builtin_amdgcn_sched_barrier(0);
                read(i + 1 < total ? i + 1 : i, 0, p0, q0); // the last one's is not used
                multiply(p1, q1);
                weave();
            }
        }
    } else {
        for (int i = 0; i < S::BUFS - 1 && i < total; ++i)
            load(i);
        for (int i = 0; i < total; ++i) {
            // this step's tile has arrived once at most the later steps' loads are out
            if (i + S::BUFS - 2 < total)
                wait_loads<(S::BUFS - 2) * (S::LP + S::LQ)>();
            else
                wait_loads<0>();
            wait_lds_and_meet();
            if (i + S::BUFS - 1 < total)
                load(i + S::BUFS - 1);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (S::TRIPLE) {
                    const lds_char *tile = (const lds_char *)smem + (i % S::BUFS) * S::stage;
                    i16x8 fp[3][S::SP], fq[3][S::SQ];
#pragma unroll
                    for (int j = 0; j < S::SQ; ++j) {
                        i16x8 three[3];
                        float_fragment<S::TQ, QK>(tile + S::at_q, at.wq * (S::SQ * 16), j, h, lane, three);
#pragma unroll
                        for (int plane = 0; plane < 3; ++plane)
                            fq[plane][j] = three[plane];
                    }
#pragma unroll
                    for (int plane = 0; plane < 3; ++plane)
                        read_p(tile + plane * (S::TP * 128), h, fp[plane]);
                    multiply(fp[0], fq[0]);
                    multiply(fp[0], fq[1]);
                    multiply(fp[1], fq[0]);
                    multiply(fp[1], fq[1]);
                    multiply(fp[0], fq[2]);
                    multiply(fp[2], fq[0]);
                } else {
                    i16x8 fp[S::SP], fq[S::SQ];
                    read(i, h, fp, fq);
                    multiply(fp, fq);
                }
            }
        }
    }
    // lane l holds, of 16 x 16 results, q = l & 15 and p = 4 (l >> 4) .. + 3; with
    // P's k contiguous, of 32 x 16, p = 8 (l >> 4) .. + 7 in two neighbours acc
    finish.template operator()<ELEM, S>(a, at, rows, acc);
}

template <class ELEM, bool PLANES, class S, class Finish>
__global__ __launch_bounds__(S::threads) void k_product(Product a, Finish finish)
{
    product<ELEM, PLANES, false, false, S>(a, finish, (int)blockIdx.x, (int)gridDim.x);
}

// --- what becomes of the results -------------------------------------------

// The class, from a lane's first, of its value i of fragment k (EIGHTS).
__device__ constexpr int class_of(int k, int i) { return (k >> 1) * 32 + (k & 1) * 4 + i; }

// Forward: per row (q) the maximum and the sum of exp(z - max) over a wave's
// classes (p), without the target's, whose logit is kept apart. Logits are in
// units of log 2 from here on, z = acc * scale2, and exp2 is the instruction, whose
// results are off by a step. Per logit a maximum, a multiply-add, an exponential and
// a sum; which class is a row's target is asked only in waves whose classes hold one,
// which classes are there at all only in the last tile.
struct FinishStats {
    Targets target; // [samples * rows]
    float2 *part;   // [parts][samples * rows]
    float *picked;  // [samples * rows]
    int *ticket;    // cleared for k_ce_rows
    float scale2;
    template <class S> struct Rows {
        int target[S::SQ];
    };
    template <class S> __device__ __forceinline__ void fetch(const Product &a, const Place &at, Rows<S> &r) const
    {
#pragma unroll
        for (int j = 0; j < S::SQ; ++j) {
            const int t = at.q0 + at.wq * (S::SQ * 16) + j * 16 + (at.lane & 15);
            r.target[j] = t < a.q.rows ? target[(int64_t)at.sample * a.q.rows + t] : kIgnored;
        }
    }
    template <class ELEM, class S>
    __device__ __forceinline__ void operator()(const Product &a, const Place &at, const Rows<S> &r,
                                               f32x4 (&acc)[S::SP][S::SQ]) const
    {
        if (blockIdx.x == 0 && threadIdx.x == 0)
            *ticket = 0;
        if (scale2 >= 0.0f)
            reduce<S, true>(a, at, r, acc);
        else
            reduce<S, false>(a, at, r, acc);
    }
    template <class S, bool POSITIVE>
    __device__ __forceinline__ void reduce(const Product &a, const Place &at, const Rows<S> &r,
                                           f32x4 (&acc)[S::SP][S::SQ]) const
    {
        constexpr float none = POSITIVE ? -kInf : kInf;
        const auto further = [](float x, float y) { return POSITIVE ? fmaxf(x, y) : fminf(x, y); };
        const int g = at.lane >> 4;
        const int w0 = at.p0 + at.wp * (S::SP * 16), v0 = w0 + 8 * g;
        const int64_t total = (int64_t)a.samples * a.q.rows;
        const bool edge = w0 + S::SP * 16 > a.p.rows;
#pragma unroll
        for (int j = 0; j < S::SQ; ++j) {
            const int t = at.q0 + at.wq * (S::SQ * 16) + j * 16 + (at.lane & 15);
            const int64_t row = (int64_t)at.sample * a.q.rows + t;
            const bool in = t < a.q.rows;
            const int d = r.target[j] - v0;
            if (edge) {
#pragma unroll
                for (int k = 0; k < S::SP; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        acc[k][j][i] = v0 + class_of(k, i) >= a.p.rows ? none : acc[k][j][i];
            }
            if (__any(d >= 0 && d < S::SP * 16)) {
                float z = 0.0f;
#pragma unroll
                for (int k = 0; k < S::SP; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool hit = d == class_of(k, i);
                        z = hit ? acc[k][j][i] : z;
                        acc[k][j][i] = hit ? none : acc[k][j][i];
                    }
                if (d >= 0 && d < S::SP * 16 && (d & 31) < 8) // the lane's own classes
                    picked[row] = z * scale2;
            }
            float m = none;
#pragma unroll
            for (int k = 0; k < S::SP; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    m = further(m, acc[k][j][i]);
            m = further(m, __shfl_xor(m, 16));
            m = further(m, __shfl_xor(m, 32));
            const float top = m == none ? -kInf : m * scale2;
            const float base = top == -kInf ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < S::SP; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    sum += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[k][j][i], scale2, -base));
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (in && g == 0)
                part[(int64_t)(at.p0 / S::TP * S::WP + at.wp) * total + row] = make_float2(top, sum);
            __builtin_amdgcn_sched_barrier(0); // rows side by side would not fit the registers
        }
    }
};

// What the backward pass needs of a row: the logits' gradient is
// fac exp2(z - top), or at_target for the target's class, in units of `unit`;
// fac 0: an ignored row or one of no upstream gradient, with top 0, since its z are
// taken as 0 (an ignored row's may be NaN) and exp2(0 - top) is infinite for a row
// whose logits all lie below -128 log 2.
struct CeCoef {
    float top, fac, at_target, unit;
};
// The units' common part, and the one that w's gradient is summed in: every unit is
// the first times a power of two.
struct CeTop {
    float unit, top;
};

// Backward: the logits' gradient of a piece, rounded to the operands' type (the
// products that follow take 16-bit operands; each value is off by half a step of
// its own size at most, as the operands x and w themselves are), or for float32 in
// three planes or as it is.
enum class Stored { narrow, planes, whole };
template <Stored AS> struct FinishGrad {
    Targets target;
    const CeCoef *coef;
    int64_t row0;        // the piece's first row
    uint16_t *g;         // [samples of the piece][rows_pad][ld] (whole: of float32)
    int64_t plane;
    float scale2;
    int rows_pad, ld, class0;
    template <class S> struct Rows {
        float top[S::SQ], fac[S::SQ];
        int target[S::SQ];
    };
    template <class S> __device__ __forceinline__ void fetch(const Product &a, const Place &at, Rows<S> &r) const
    {
#pragma unroll
        for (int j = 0; j < S::SQ; ++j) {
            const int t = at.q0 + at.wq * (S::SQ * 16) + j * 16 + (at.lane & 15);
            const int64_t row = row0 + (int64_t)at.sample * a.q.rows + t;
            r.top[j] = r.fac[j] = 0.0f;
            r.target[j] = kIgnored;
            if (t < a.q.rows) {
                r.top[j] = coef[row].top;
                r.fac[j] = coef[row].fac;
                r.target[j] = target[row] - class0;
            }
        }
    }
    template <class ELEM, class S>
    __device__ __forceinline__ void operator()(const Product &a, const Place &at, const Rows<S> &r,
                                               f32x4 (&acc)[S::SP][S::SQ]) const
    {
        constexpr int W = S::SP * 16, LD = W + 8; // a row of the wave's results in shared memory
        static_assert(16 * LD * 2 <= S::lds / S::waves, "a wave's part of the tiles holds 16 rows");
        wait_lds_and_meet();
        const int w0 = at.p0 + at.wp * W, v0 = w0 + 8 * (at.lane >> 4);
        const bool edge = w0 + W > a.p.rows;
#pragma unroll
        for (int j = 0; j < S::SQ; ++j) {
            const int t = at.q0 + at.wq * (S::SQ * 16) + j * 16 + (at.lane & 15);
            const float top = r.top[j], fac = r.fac[j];
            const int d = r.target[j] - v0;
            if (__any(fac == 0.0f)) {
#pragma unroll
                for (int k = 0; k < S::SP; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        acc[k][j][i] = fac == 0.0f ? 0.0f : acc[k][j][i];
            }
#pragma unroll
            for (int k = 0; k < S::SP; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[k][j][i] = fac * __builtin_amdgcn_exp2f(__builtin_fmaf(acc[k][j][i], scale2, -top));
            const bool here = d >= 0 && d < S::SP * 16;
            if (__any(here)) {
                const float mine = here ? coef[row0 + (int64_t)at.sample * a.q.rows + t].at_target : 0.0f;
#pragma unroll
                for (int k = 0; k < S::SP; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        acc[k][j][i] = d == class_of(k, i) ? mine : acc[k][j][i];
            }
            if (edge) {
#pragma unroll
                for (int k = 0; k < S::SP; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        acc[k][j][i] = v0 + class_of(k, i) >= a.p.rows ? 0.0f : acc[k][j][i];
            }
            const int q0 = at.q0 + at.wq * (S::SQ * 16) + j * 16;
            const int64_t first = ((int64_t)at.sample * rows_pad + q0) * ld + w0;
            uint16_t *to = g + first;
            const auto write = [&](auto values, uint16_t *out) {
#pragma unroll
                for (int k = 0; k < S::SP; k += 2) {
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        v[i] = acc[k + (i >> 2)][j][i & 3];
                    *(lds_ptr<i16x8>)(at.lds + ((at.lane & 15) * LD + k * 16 + 8 * (at.lane >> 4)) * 2) = values(v);
                }
                wave_lds();
                const int n = min(16, rows_pad - q0) * (W / 8);
#pragma unroll
                for (int u = 0; u < W / 32; ++u) {
                    const int i = at.lane + u * 64, r = i / (W / 8), c = i % (W / 8) * 8;
                    if (i < n && w0 + c < ld)
                        *(i16x8 *)(out + (int64_t)r * ld + c) = *(lds_ptr<i16x8>)(at.lds + (r * LD + c) * 2);
                }
                wave_lds();
            };
            if constexpr (AS == Stored::whole) {
                constexpr int LF = W + 4;
                static_assert(16 * LF * 4 <= S::lds / S::waves, "a wave's part of the tiles holds 16 rows");
                const auto row = (lds_ptr<float>)at.lds;
#pragma unroll
                for (int k = 0; k < S::SP; ++k)
                    *(lds_ptr<f32x4>)(row + (at.lane & 15) * LF + (k >> 1) * 32 + 8 * (at.lane >> 4) + (k & 1) * 4) = acc[k][j];
                wave_lds();
                const int n = min(16, rows_pad - q0) * (W / 4);
#pragma unroll
                for (int u = 0; u < W / 16; ++u) {
                    const int i = at.lane + u * 64, r = i / (W / 4), c = i % (W / 4) * 4;
                    if (i < n && w0 + c < ld)
                        *(f32x4 *)((float *)g + first + (int64_t)r * ld + c) = *(lds_ptr<f32x4>)(row + r * LF + c);
                }
                wave_lds();
            } else if constexpr (AS == Stored::planes) {
                write([](const float (&v)[8]) { return planes_of<false>(v).a; }, to);
                write([](const float (&v)[8]) { return planes_of<false>(v).b; }, to + plane);
                write([](const float (&v)[8]) { return planes_of<false>(v).c; }, to + 2 * plane);
            } else {
                write([](const float (&v)[8]) {
                    i16x8 r;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        r[i] = (short)ELEM::from(v[i]);
                    return r;
                }, to);
            }
            __builtin_amdgcn_sched_barrier(0); // rows side by side would not fit the registers
        }
    }
};

// OUT: the type of a gradient that goes out.
template <class OUT> using Element = std::conditional_t<std::is_same_v<OUT, float>, float, uint16_t>;
template <class OUT> __device__ __forceinline__ Element<OUT> element(float v)
{
    if constexpr (std::is_same_v<OUT, float>)
        return v;
    else
        return OUT::from(v);
}
// Neighbours at any element.
template <class T, int N> struct __attribute__((packed, aligned(sizeof(T)))) Loose {
    T v[N];
};

// What the rounding of the targets' entries took from x's gradient: a row's entry
// for its target is as large as all the others together, so that its half step
// was most of the gradient's error (4 x 4769 x 4507 x 64 bfloat16: 1.5 times that of
// one rounding at the end, now 1.0). It goes back in as rest w_target; the gradient
// of w, where a class adds up many rows' entries, goes without.
template <class OUT> struct TargetRest {
    Targets target;
    const uint16_t *w;   // [samples][classes][dim] as the caller holds it
    const CeCoef *coef;
    int64_t row0;        // the rows of w's first sample begin here in target
    int rows, dim;       // per sample
    float inv_unit;
    // v[u] += rest w_target[c + u] for u < n of row `row` from row0 on
    template <int N> __device__ __forceinline__ void add(int64_t row, int c, int n, float (&v)[N]) const
    {
        const float entry = coef[row].at_target;
        const float rest = (entry - OUT::to(OUT::from(entry))) * coef[row].unit * inv_unit;
        const int t = target[row0 + row];
        if (t < 0 || rest == 0.0f || !(fabsf(rest) < kInf)) // beyond float16's range the entry is infinite
            return;
        const uint16_t *from = w + (row / rows * target.classes + t) * dim + c;
        if (n >= N) {
            const Loose<uint16_t, N> x = *(const Loose<uint16_t, N> *)from;
#pragma unroll
            for (int u = 0; u < N; ++u)
                v[u] = __builtin_fmaf(rest, OUT::to(x.v[u]), v[u]);
        } else {
            for (int u = 0; u < n; ++u)
                v[u] = __builtin_fmaf(rest, OUT::to(from[u]), v[u]);
        }
    }
};
template <> struct TargetRest<float> { // all bits are kept
    Targets target;
    const uint16_t *w;
    const CeCoef *coef;
    int64_t row0;
    int rows, dim;
    float inv_unit;
    template <int N> __device__ __forceinline__ void add(int64_t, int, int, float (&)[N]) const {}
};

// A gradient [samples][q rows][p rows]: rounded once and stored, times a factor
// per row (coef) or for all (top).
template <class OUT> struct FinishStore {
    void *out;
    TargetRest<OUT> rest; // grad_x
    const CeCoef *coef; // grad_x: the rows' units, else NULL
    const CeTop *top;   // grad_w: the largest unit
    float inv_unit;     // 1 / ELEM::kUnit
    int64_t sample;     // elements from one sample's output to the next
    template <class S> struct Rows {};
    template <class S> __device__ __forceinline__ void fetch(const Product &, const Place &, Rows<S> &) const {}
    template <class ELEM, class S>
    __device__ __forceinline__ void operator()(const Product &a, const Place &at, const Rows<S> &,
                                               f32x4 (&acc)[S::SP][S::SQ]) const
    {
        float unit[S::SQ];
#pragma unroll
        for (int j = 0; j < S::SQ; ++j) {
            const int q = min(at.q0 + at.wq * (S::SQ * 16) + j * 16 + (at.lane & 15), a.q.rows - 1);
            unit[j] = (coef ? coef[(int64_t)at.sample * a.q.rows + q].unit : top->top) * inv_unit;
        }
        // 16 rows at a time pass through shared memory, from where a wave writes
        // whole pieces of each row, 16 bytes a lane wherever the row begins (a
        // global store needs no more alignment than its elements).
        constexpr int VEC = 16 / sizeof(Element<OUT>);
        constexpr int W = S::SP * 16, LD = W + 4; // a row of the wave's results, in float32
        static_assert(16 * LD * 4 <= S::lds / S::waves, "a wave's part of the tiles holds 16 rows");
        wait_lds_and_meet();
        const auto row = (lds_ptr<float>)at.lds;
        const int p0 = at.p0 + at.wp * W, q0 = at.q0 + at.wq * (S::SQ * 16);
#pragma unroll
        for (int j = 0; j < S::SQ; ++j) {
#pragma unroll
            for (int k = 0; k < S::SP; ++k)
                *(lds_ptr<f32x4>)(row + (at.lane & 15) * LD + k * 16 + 4 * (at.lane >> 4)) = acc[k][j] * unit[j];
            wave_lds();
            const int n = min(16, a.q.rows - q0 - j * 16) * (W / VEC);
            const int64_t to = at.sample * sample + (int64_t)(q0 + j * 16) * a.p.rows + p0;
            for (int i = at.lane; i < n; i += 64) {
                const int r = i / (W / VEC), c = i % (W / VEC) * VEC, left = a.p.rows - p0 - c;
                const lds_ptr<float> from = row + r * LD + c;
                auto *at_out = (Element<OUT> *)out + to + (int64_t)r * a.p.rows + c;
                float x[VEC];
#pragma unroll
                for (int u = 0; u < VEC; ++u)
                    x[u] = from[u];
                if (coef)
                    rest.add((int64_t)at.sample * a.q.rows + q0 + j * 16 + r, p0 + c, left, x);
                Loose<Element<OUT>, VEC> v;
#pragma unroll
                for (int u = 0; u < VEC; ++u)
                    v.v[u] = element<OUT>(x[u]);
                if (left >= VEC) {
                    *(Loose<Element<OUT>, VEC> *)at_out = v;
                } else {
#pragma unroll
                    for (int u = 0; u < VEC; ++u)
                        if (u < left)
                            at_out[u] = v.v[u];
                }
            }
            wave_lds();
        }
    }
};

// One part of a gradient's sum, in float32 [split][samples][q rows][ld]; added
// to what an earlier piece left there.
struct FinishPart {
    float *part;
    int64_t split, sample; // elements from one part, one sample to the next
    int ld;                // p rows up to a multiple of 4
    bool add;
    template <class S> struct Rows {};
    template <class S> __device__ __forceinline__ void fetch(const Product &, const Place &, Rows<S> &) const {}
    template <class ELEM, class S>
    __device__ __forceinline__ void operator()(const Product &a, const Place &at, const Rows<S> &,
                                               f32x4 (&acc)[S::SP][S::SQ]) const
    {
        const int p0 = at.p0 + at.wp * (S::SP * 16) + 4 * (at.lane >> 4);
#pragma unroll
        for (int j = 0; j < S::SQ; ++j) {
            const int q = at.q0 + at.wq * (S::SQ * 16) + j * 16 + (at.lane & 15);
            if (q >= a.q.rows)
                continue;
            float *to = part + at.split * split + at.sample * sample + (int64_t)q * ld;
#pragma unroll
            for (int k = 0; k < S::SP; ++k) {
                const int p = p0 + k * 16;
                if (p < ld) {
                    f32x4 v = acc[k][j];
                    if (add)
                        v += *(f32x4 *)(to + p);
                    *(f32x4 *)(to + p) = v;
                }
            }
        }
    }
};

// A gradient whole or in parts.
template <class OUT> struct FinishOut {
    FinishStore<OUT> store;
    FinishPart part;
    bool in_parts;
    template <class S> struct Rows {};
    template <class S> __device__ __forceinline__ void fetch(const Product &, const Place &, Rows<S> &) const {}
    template <class ELEM, class S>
    __device__ __forceinline__ void operator()(const Product &a, const Place &at, const Rows<S> &,
                                               f32x4 (&acc)[S::SP][S::SQ]) const
    {
        if (in_parts)
            part.template operator()<ELEM, S>(a, at, FinishPart::Rows<S>{}, acc);
        else
            store.template operator()<ELEM, S>(a, at, typename FinishStore<OUT>::template Rows<S>{}, acc);
    }
};

template <class OUT> struct GradJob {
    Product a;
    FinishOut<OUT> out;
    int blocks; // 0: not wanted
};

// Both gradients of a piece, x's [rows][dim] = G [rows][classes] w [classes][dim]
// and w's [classes][dim] = G^T [classes][rows] x [rows][dim], in one launch: each
// alone often leaves compute units without a tile, or in a last round with few.
template <class ELEM, bool PLANES, class S, class OUT>
__global__ __launch_bounds__(S::threads) void k_gradients(GradJob<OUT> x, GradJob<OUT> w, bool w_first)
{
    const int first = w_first ? w.blocks : x.blocks;
    const bool second = (int)blockIdx.x >= first;
    const int block = (int)blockIdx.x - (second ? first : 0);
    if (second != w_first)
        product<ELEM, PLANES, true, true, S>(w.a, w.out, block, w.blocks);
    else
        product<ELEM, PLANES, true, false, S>(x.a, x.out, block, x.blocks);
}

// ---------------------------------------------------------------------------
// the kernels around the products
// ---------------------------------------------------------------------------

// The upstream gradient of row i, times the logits' scale.
struct Upstream {
    const float *grad_loss, *total;
    int reduction;
    float scale;
    __device__ __forceinline__ float operator()(int64_t i) const
    {
        const float g = grad_loss[reduction == 0 ? i : 0];
        return (reduction == 2 ? g / total[1] : g) * scale;
    }
};

// The largest |b| over the rows that count, of upstream gradients b, the largest
// size |b| + |c| with the penalty's part c = 2 z_weight lse b, and the largest
// size times a feature of its row.
struct Largest {
    float b, size, x;
    __device__ __forceinline__ void join(const Largest &o)
    {
        b = fmaxf(b, o.b);
        size = fmaxf(size, o.size);
        x = fmaxf(x, o.x);
    }
    // over the workgroup, in its first thread (whole: in all of them)
    __device__ __forceinline__ void join_all(Largest *sm, bool whole)
    {
        for (int o = 32; o > 0; o >>= 1)
            join(Largest{__shfl_xor(b, o), __shfl_xor(size, o), __shfl_xor(x, o)});
        if (lane_id() == 0)
            sm[threadIdx.x >> 6] = *this;
        __syncthreads();
        if (whole || threadIdx.x == 0)
            for (int w = 0; w < kBlock / 64; ++w)
                join(sm[w]);
    }
};

// FEATURES: with the float16 features x [n][dim], `lanes` lanes a row (1777 x
// 1003: 5 us, 8192 x 1024: 9 us, 200000 x 64: 17 us), else one (5 us).
template <bool FEATURES>
__global__ __launch_bounds__(kBlock) void k_ce_size(const CeRow *rows, Targets target, Upstream up, float z_weight,
                                                    int64_t n, const uint16_t *x, int dim, int lanes, Largest *block_top)
{
    __shared__ Largest sm[kBlock / 64];
    Largest m{0.0f, 0.0f, 0.0f};
    const int per = FEATURES ? lanes : 1, lane = threadIdx.x & (per - 1);
    for (int64_t i = ((int64_t)blockIdx.x * kBlock + threadIdx.x) / per; i < n; i += (int64_t)gridDim.x * (kBlock / per)) {
        const float b = up(i), size = fabsf(b) + (z_weight != 0.0f ? fabsf(2.0f * z_weight * rows[i].lse * b) : 0.0f);
        if (target[i] == kIgnored || !(size < kInf))
            continue;
        float feature = 0.0f;
        if constexpr (FEATURES) {
            const uint16_t *row = x + i * dim;
            for (int c = lane * 8; c < dim; c += per * 8) {
                if (c + 8 <= dim) {
                    const Loose<uint16_t, 8> v = *(const Loose<uint16_t, 8> *)(row + c);
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        feature = fmaxf(feature, fabsf(F16::to(v.v[u])));
                } else {
                    for (int u = c; u < dim; ++u)
                        feature = fmaxf(feature, fabsf(F16::to(row[u])));
                }
            }
        }
        m.join(Largest{fabsf(b), size, fminf(feature * size, FLT_MAX)});
    }
    m.join_all(sm, false);
    if (threadIdx.x == 0)
        block_top[blockIdx.x] = m;
}

// The smallest e with size <= unit 2^e, within [-60, 20].
__device__ __forceinline__ int exponent_over(float size, float unit)
{
    int e = 0;
    const float f = frexpf(size / unit, &e); // in [1/2, 1)
    if (f == 0.5f)
        --e;
    return size > 0.0f ? min(max(e, -60), 20) : -60;
}

// The backward pass's coefficients of a row. Its gradient is stored in units of
// the largest upstream gradient times a power of two, so that it lies in
// [-1, 1] and equal upstream gradients (a mean) cost the target's value -miss no
// rounding of their own. tops: k_ce_size's, or 0 of them where all rows have the
// same upstream gradient and no penalty.
struct Coefs {
    const CeRow *rows;
    Targets target;
    Upstream up;
    float z_weight, stored_unit;
    const Largest *block_top;
    int tops;
    // by the whole workgroup
    __device__ __forceinline__ CeTop top() const
    {
        Largest m{0.0f, 0.0f, 0.0f};
        if (tops == 0) {
            m.b = m.size = fabsf(up(0));
        } else {
            __shared__ Largest sm[kBlock / 64];
            for (int i = threadIdx.x; i < tops; i += kBlock)
                m.join(block_top[i]);
            m.join_all(sm, true);
        }
        // within 2^+-60: its smallest and largest multiples stay normal
        const float unit = m.b >= 0x1p-60f && m.b <= 0x1p60f ? m.b : 1.0f;
        const float top = ldexpf(unit, max(exponent_over(m.size, unit), 0));
        // A row's unit is less than twice its size, so that its features times its
        // unit over the one given here stay below 2^15 where m.x is known.
        const int shift = m.x > 0.0f ? min(max(14 - exponent_over(m.x, top), 0), 40) : 0;
        return CeTop{unit, ldexpf(top, -shift)};
    }
    __device__ __forceinline__ CeCoef operator()(int64_t i, const CeTop &t) const
    {
        const int at = target[i];
        if (at == kIgnored)
            return CeCoef{0.0f, 0.0f, 0.0f, t.unit};
        const CeRow r = rows[i];
        const float b = up(i), c = z_weight != 0.0f ? 2.0f * z_weight * r.lse * b : 0.0f;
        const float size = fabsf(b) + fabsf(c);
        const float mine = ldexpf(t.unit, size < kInf ? exponent_over(size, t.unit) : 0);
        const float bn = b / mine * stored_unit, cn = c / mine * stored_unit;
        CeCoef k{r.top, (bn + cn) * r.inv_total, cn * (1.0f - r.miss) - bn * r.miss, mine};
        if (at == kOutside)
            k.fac = __builtin_nanf("");
        if (k.fac == 0.0f)
            k.top = 0.0f;
        return k;
    }
};

// Rows copied to dim_pad columns (zeros behind dim) and, where scaled, rows_out
// rows a sample with every row times its unit over that of w's gradient (a power of
// two; zero for ignored rows, whatever they hold). Rows of equal weight stay as they
// are; of others the largest product of a feature and its row's weight lies above
// 2^13 in float16, so that features down to 2^-27 of it keep all their bits and
// smaller ones are off by 2^-38 of it at most. In the backward
// pass the first coef_blocks workgroups write the rows' coefficients. Bound by
// memory (50001 x 1003 to 50001 x 1024 half precision, 203 MB: 45 us, 4.5 TB/s).
template <class IN> __device__ __forceinline__ float get(const void *in, int64_t at) { return IN::to(((const uint16_t *)in)[at]); }
template <> __device__ __forceinline__ float get<float>(const void *in, int64_t at) { return ((const float *)in)[at]; }

struct PackJob {
    const void *in;
    uint16_t *out;
    int64_t n;           // elements of one plane of out
    int rows, rows_out;  // per sample
    bool scaled;
    unsigned blocks;
};
constexpr int kPackJobs = 3;
struct PackJobs {
    PackJob job[kPackJobs];
    int dim, dim_pad;
    unsigned coef_blocks;
    int64_t coef_rows;
    Coefs coefs;
    CeCoef *coef;
    CeTop *top;
};

template <class IN> __global__ __launch_bounds__(kBlock) void k_ce_pack(PackJobs jobs)
{
    unsigned block = blockIdx.x;
    if (block < jobs.coef_blocks) {
        const CeTop top = jobs.coefs.top();
        if (block == 0 && threadIdx.x == 0)
            *jobs.top = top;
        const int64_t i = (int64_t)block * kBlock + threadIdx.x;
        if (i < jobs.coef_rows)
            jobs.coef[i] = jobs.coefs(i, top);
        return;
    }
    block -= jobs.coef_blocks;
    int which = 0;
    while (block >= jobs.job[which].blocks)
        block -= jobs.job[which++].blocks;
    const PackJob &p = jobs.job[which];
    CeTop top{1.0f, 1.0f};
    if (p.scaled)
        top = jobs.coefs.top();
    const int64_t i = ((int64_t)block * kBlock + threadIdx.x) * 8;
    if (i >= p.n)
        return;
    const int64_t r = i / jobs.dim_pad;
    const int d = (int)(i - r * jobs.dim_pad);
    const int64_t sample = r / p.rows_out;
    const int t = (int)(r - sample * p.rows_out);
    float f = 1.0f;
    bool keep = t < p.rows;
    const int64_t row = sample * p.rows + t;
    if (p.scaled && keep) {
        keep = jobs.coefs.target[row] != kIgnored;
        f = keep ? jobs.coefs(row, top).unit / top.top : 0.0f;
    }
    float v[8];
    const int64_t at = row * jobs.dim + d;
    constexpr int size = std::is_same_v<IN, float> ? 4 : 2;
    if (keep && d + 8 <= jobs.dim) {
        // eight neighbours wherever they lie: a global load of 16 bytes needs no
        // more alignment than its elements (50001 x 1003 half precision: 2.5 TB/s
        // element by element)
        if constexpr (size == 4) {
            const Loose<float, 8> raw = *(const Loose<float, 8> *)((const float *)p.in + at);
#pragma unroll
            for (int u = 0; u < 8; ++u)
                v[u] = raw.v[u] * f;
        } else {
            const Loose<uint16_t, 8> raw = *(const Loose<uint16_t, 8> *)((const uint16_t *)p.in + at);
#pragma unroll
            for (int u = 0; u < 8; ++u)
                v[u] = IN::to(raw.v[u]) * f;
        }
    } else {
#pragma unroll
        for (int u = 0; u < 8; ++u)
            v[u] = keep && d + u < jobs.dim ? get<IN>(p.in, at + u) * f : 0.0f;
    }
    i16x8 p0;
    if constexpr (size == 4) {
        const Planes x = planes_of<true>(v);
        p0 = x.a;
        *(i16x8 *)(p.out + p.n + i) = x.b;
        *(i16x8 *)(p.out + 2 * p.n + i) = x.c;
    } else {
#pragma unroll
        for (int u = 0; u < 8; ++u)
            p0[u] = (short)IN::from(v[u]);
    }
    *(i16x8 *)(p.out + i) = p0;
}

// What the workgroups of k_ce_rows leave for the last of them.
struct LossSum {
    double sum;
    int64_t count;
};

// Joins a row's parts (65536 rows of 128 parts, 67 MB: 27 us; 8192 rows of 1024:
// 20 us), and the rows' losses. The last sums are in double precision. A workgroup takes kBlock / THREADS
// rows; thread k of a row takes its parts k, k + THREADS, ... The last workgroup
// to end adds up the sums of all of them, in their order.
template <int THREADS>
__global__ __launch_bounds__(kBlock) void k_ce_rows(const float2 *part, int parts, const float *picked, Targets target,
                                                    int64_t n, float z_weight, int reduction, float *row_loss, CeRow *rows,
                                                    LossSum *sums, int *ticket, float *loss, float *total)
{
    constexpr int ROWS = kBlock / THREADS;
    __shared__ float2 sm[THREADS][ROWS + 1];
    __shared__ LossSum sl[ROWS];
    __shared__ bool is_last;
    const int r = threadIdx.x % ROWS, k0 = threadIdx.x / ROWS;
    const int64_t row = (int64_t)blockIdx.x * ROWS + r;
    float m = -kInf, sum = 0.0f;
    if (row < n) {
        constexpr int U = THREADS == 4 ? 16 : 8; // loads in flight
        for (int k = k0; k < parts; k += THREADS * U) {
            float2 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = k + u * THREADS;
                v[u] = at < parts ? part[(int64_t)at * n + row] : make_float2(-kInf, 0.0f);
            }
            float top = m;
#pragma unroll
            for (int u = 0; u < U; ++u)
                top = fmaxf(top, v[u].x);
            const float base = top == -kInf ? 0.0f : top;
            sum *= __builtin_amdgcn_exp2f(m - base);
#pragma unroll
            for (int u = 0; u < U; ++u)
                sum = __builtin_fmaf(v[u].y, __builtin_amdgcn_exp2f(v[u].x - base), sum);
            m = top;
        }
    }
    sm[k0][r] = make_float2(m, sum);
    __syncthreads();
    constexpr int LEFT = THREADS < 16 ? THREADS : 16;
    if constexpr (THREADS > 16) { // 16 are left, each with a fixed share
        if (k0 < 16) {
            float top = m;
            for (int k = k0 + 16; k < THREADS; k += 16)
                top = fmaxf(top, sm[k][r].x);
            const float base = top == -kInf ? 0.0f : top;
            sum *= __builtin_amdgcn_exp2f(m - base);
            for (int k = k0 + 16; k < THREADS; k += 16)
                sum = __builtin_fmaf(sm[k][r].y, __builtin_amdgcn_exp2f(sm[k][r].x - base), sum);
            sm[k0][r] = make_float2(top, sum);
        }
        __syncthreads();
    }
    if (threadIdx.x < ROWS) {
        LossSum mine_sum{0.0, 0};
        if (row < n) {
            const int t = target[row];
            const float z = t >= 0 ? picked[row] : -kInf;
            float top = z;
            for (int k = 0; k < LEFT; ++k)
                top = fmaxf(top, sm[k][r].x);
            const float base = top == -kInf ? 0.0f : top;
            double others = 0.0;
            for (int k = 0; k < LEFT; ++k)
                others += (double)sm[k][r].y * (double)exp2f(sm[k][r].x - base);
            const double mine = t >= 0 ? (double)exp2f(z - base) : 0.0;
            const double all = others + mine;
            const double lse = (double)base * M_LN2 + log(all);
            double l = mine > 0.5 ? log1p(others / mine) : lse - (double)z * M_LN2;
            float miss = (float)(others / all);
            if (z_weight != 0.0f)
                l += (double)z_weight * lse * lse;
            if (t == kIgnored)
                l = 0.0;
            if (t == kOutside)
                l = miss = __builtin_nanf("");
            mine_sum = {l, t != kIgnored};
            if (reduction == 0)
                row_loss[row] = (float)l;
            if (rows)
                rows[row] = CeRow{top, (float)(1.0 / all), miss, (float)lse};
        }
        sl[r] = mine_sum;
    }
    if (reduction == 0)
        return;
    __syncthreads();
    if (threadIdx.x == 0) {
        LossSum s = sl[0];
#pragma unroll 8
        for (int k = 1; k < ROWS; ++k) {
            s.sum += sl[k].sum;
            s.count += sl[k].count;
        }
        // device-scope stores and loads go past the XCDs' own L2s, so a wait for
        // the stores is all the order that the ticket needs (a release fence
        // would write the whole L2 back: 10 us more for 512 workgroups)
        __hip_atomic_store(&sums[blockIdx.x].sum, s.sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(&sums[blockIdx.x].count, s.count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        is_last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (!is_last)
        return;
    __shared__ double ds[kBlock / 64];
    __shared__ int64_t dc[kBlock / 64];
    double a = 0.0;
    int64_t c = 0;
    for (unsigned i = threadIdx.x; i < gridDim.x; i += kBlock) {
        a += __hip_atomic_load(&sums[i].sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        c += __hip_atomic_load(&sums[i].count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    a = wave_sum(a);
    for (int o = 32; o > 0; o >>= 1)
        c += __shfl_xor(c, o);
    if (lane_id() == 0) {
        ds[threadIdx.x >> 6] = a;
        dc[threadIdx.x >> 6] = c;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kBlock / 64; ++w) {
            a += ds[w];
            c += dc[w];
        }
        const double counted = c > 1 ? (double)c : 1.0;
        loss[0] = (float)(reduction == 2 ? a / counted : a);
        if (total) {
            total[0] = (float)a;
            total[1] = (float)counted;
        }
    }
}

// Adds up the parts of a gradient and rounds it; one gradient or both (8192 x 4096
// in one part: 38 us, 5 TB/s).
struct JoinJob {
    const float *part;
    void *out;
    int64_t rows, split; // elements from one part to the next
    int splits;
    const CeCoef *coef;  // grad_x: the rows' units, else NULL
    unsigned blocks;
};
template <class OUT> struct JoinJobs {
    JoinJob job[2];
    TargetRest<OUT> rest;
    int cols, ld;
    const CeTop *top;
    float inv_unit;
};
template <class OUT> __global__ __launch_bounds__(kBlock) void k_ce_join(JoinJobs<OUT> jobs)
{
    const bool second = blockIdx.x >= jobs.job[0].blocks;
    const JoinJob &p = jobs.job[second];
    const int64_t i = ((int64_t)(blockIdx.x - (second ? jobs.job[0].blocks : 0)) * kBlock + threadIdx.x) * 4;
    const int64_t r = i / jobs.ld;
    const int c = (int)(i - r * jobs.ld);
    if (r >= p.rows)
        return;
    f32x4 v = *(const f32x4 *)(p.part + i);
    for (int s = 1; s < p.splits; ++s)
        v += *(const f32x4 *)(p.part + s * p.split + i);
    v *= (p.coef ? p.coef[r].unit : jobs.top->top) * jobs.inv_unit;
    float x[4] = {v[0], v[1], v[2], v[3]};
    if (p.coef)
        jobs.rest.add(r, c, jobs.cols - c, x);
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (c + u < jobs.cols)
            ((Element<OUT> *)p.out)[r * jobs.cols + c + u] = element<OUT>(x[u]);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------

using Large = Shape<256, 256, 2, 4, 2, true>; // products over the features: fewer reductions over the classes
using Tall = Shape<256, 256, 4, 2, 2, true>;  // the gradients' (8192 x 4096 x 8192: 386 us; its transpose 394)
using Medium = Shape<128, 128, 2, 2, 2>;
using Narrow = Shape<128, 16, 4, 1, 4>;
using Thin = Shape<64, 128, 2, 2, 2>;
using ThinTriple = Shape<64, 128, 2, 4, 2, false, true>; // 16 of 2048 x 2048 x 64: 156 us, with Q in planes 170

int ceil_to(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }
int64_t pad_to(int64_t a, int64_t b) { return (a + b - 1) / b * b; }

enum class Kind { large, medium, narrow, thin };

// Whether 256 x 256 tiles, one a compute unit, end before 128 x 128 ones, two a
// compute unit: rounds of each, a round of the latter taking 0.58 of the former's
// time (8192 x 8192 x 1024: 116 us against 134 in four rounds and eight).
constexpr double kMediumRound = 0.58;
bool large_tiles(int64_t p, int64_t q, int64_t batches)
{
    const int64_t large = ceil_to(p, 256) * (int64_t)ceil_to(q, 256) * batches;
    const int64_t medium = ceil_to(p, 128) * (int64_t)ceil_to(q, 128) * batches;
    return ceil_to(large, 256) <= kMediumRound * ceil_to(medium, 512);
}

// The tile of a product of p classes and q rows, `batches` of them. Forward, 16
// rows where there are no more (one row of 131072 x 4096 195 us, of 32000 x 4096
// 46; in tiles of 128 206 and 65); backward the logits' gradient is written for
// whole steps of rows.
Kind choose(int64_t p, int64_t q, int64_t batches, bool forward)
{
    if (forward && q <= 16)
        return Kind::narrow;
    return large_tiles(p, q, batches) ? Kind::large : Kind::medium;
}
// The tile and the parts of the gradients' launch, whose p axis is the features:
// x's sums run over steps_x steps of classes, w's over steps_w of rows, and may be
// cut into parts. No more than 64 features would leave half of a 128 wide tile
// empty; else the tile and the parts that end first, in steps of the large tile:
// the workgroups' steps as they follow each other on the compute units, and each
// part's results written and read again in float32 (at about 4 TB/s, 6 MB a step).
struct Cut {
    Kind kind;
    int split_x, split_w;
    bool w_first; // the side with the longer workgroups
};
// When n1 jobs of d1 steps and then n2 of d2 end on so many slots.
double end_of(int64_t n1, double d1, int64_t n2, double d2, int64_t slots)
{
    const int64_t rounds = n1 / slots, last = n1 % slots;
    const double t = (double)rounds * d1, one = t + (last ? d1 : 0.0);
    if (n2 == 0)
        return one;
    const double k = (double)ceil_to(n2, slots - last); // rounds of the slots that are free first
    if (k * d2 <= d1 || last == 0)
        return std::max(one, t + k * d2);
    return t + std::ceil(((double)n2 + (double)last * (d1 / d2)) / (double)slots) * d2;
}
Cut choose_grads(int64_t dim, int64_t rows, int64_t classes, int64_t batches, int64_t steps_x, int64_t steps_w,
                 int planes, bool want_x, bool want_w)
{
    static constexpr int cuts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
    const int64_t least = planes > 1 ? 2 : 8; // a float32 step is six
    const double each = planes > 1 ? kPlaneProducts : 1;
    Cut best{Kind::medium, 1, 1, false};
    double least_cost = HUGE_VAL;
    // slots: workgroups that run at once; round: their step's time
    const auto consider = [&](Kind kind, int tile_p, int tile_q, int64_t slots, double round) {
        const int64_t x = want_x ? ceil_to(dim, tile_p) * (int64_t)ceil_to(rows, tile_q) * batches : 0;
        const int64_t w = want_w ? ceil_to(dim, tile_p) * (int64_t)ceil_to(classes, tile_q) * batches : 0;
        const auto most = [&](int64_t tiles, int64_t steps) {
            return tiles ? std::max<int64_t>(1, std::min<int64_t>({2 * slots / tiles, steps / least, 64})) : 1;
        };
        const auto join = [&](int cut, int64_t q) {
            return cut > 1 ? (double)(cut + 1) * (double)(dim * q * batches) * 8.0 / 6e6 + 4.0 : 0.0;
        };
        const int64_t most_x = most(x, steps_x), most_w = most(w, steps_w);
        for (const int cx : cuts) {
            if (cx > most_x)
                break;
            const double dx = ((double)ceil_to(steps_x, cx) * each + 4.0) * round, jx = join(cx, rows);
            for (const int cw : cuts) {
                if (cw > most_w)
                    break;
                const double dw = ((double)ceil_to(steps_w, cw) * each + 4.0) * round;
                const bool w_first = dw > dx;
                const double c = (w_first ? end_of(w * cw, dw, x * cx, dx, slots) : end_of(x * cx, dx, w * cw, dw, slots)) +
                                 jx + join(cw, classes);
                if (c < least_cost) {
                    least_cost = c;
                    best = {kind, cx, cw, w_first};
                }
            }
        }
    };
    if (dim <= 64) {
        consider(Kind::thin, 64, 128, planes > 1 ? 256 : 768, planes > 1 ? 0.24 : 0.5);
    } else {
        consider(Kind::medium, 128, 128, 512, kMediumRound);
        consider(Kind::large, 256, 256, 256, 1.0);
    }
    return best;
}
int tile_p(Kind k) { return k == Kind::large ? 256 : k == Kind::thin ? 64 : 128; }
int waves_p(Kind k) { return k == Kind::narrow ? Narrow::WP : 2; }

template <class S> int cover(Product &a, int64_t p, int64_t q)
{
    a.tiles_p = ceil_to(p, S::TP);
    a.tiles_q = ceil_to(q, S::TQ);
    a.group = std::min(a.tiles_q, 8);
    return (int)((int64_t)a.tiles_p * a.tiles_q * a.samples * a.splits);
}

template <class ELEM, bool PLANES, class S, class F>
void launch_shape(Product a, int64_t cover_p, int64_t cover_q, const F &f, hipStream_t s)
{
    const int grid = cover<S>(a, cover_p, cover_q);
    (void)set_dynamic_lds((const void *)k_product<ELEM, PLANES, S, F>, S::lds);
    k_product<ELEM, PLANES, S, F><<<dim3(grid), dim3(S::threads), S::lds, s>>>(a, f);
}

template <class ELEM, bool PLANES, class F>
void launch_product(Kind kind, const Product &a, int64_t cover_p, int64_t cover_q, const F &f, hipStream_t s)
{
    if (kind == Kind::large)
        launch_shape<ELEM, PLANES, Large>(a, cover_p, cover_q, f, s);
    else if (kind == Kind::medium)
        launch_shape<ELEM, PLANES, Medium>(a, cover_p, cover_q, f, s);
    else if constexpr (std::is_same_v<F, FinishStats>)
        launch_shape<ELEM, PLANES, Narrow>(a, cover_p, cover_q, f, s);
}

template <class ELEM, bool PLANES, class OUT>
void launch_gradients(const Cut &cut, GradJob<OUT> x, GradJob<OUT> w, bool want_x, bool want_w, hipStream_t s)
{
    const auto with = [&](auto shape) {
        using S = decltype(shape);
        x.blocks = want_x ? cover<S>(x.a, x.a.p.rows, x.a.q.rows) : 0;
        w.blocks = want_w ? cover<S>(w.a, w.a.p.rows, w.a.q.rows) : 0;
        const auto k = k_gradients<ELEM, PLANES, S, OUT>;
        (void)set_dynamic_lds((const void *)k, S::lds);
        k<<<dim3(x.blocks + w.blocks), dim3(S::threads), S::lds, s>>>(x, w, cut.w_first);
    };
    if (cut.kind == Kind::large)
        with(Tall{});
    else if (cut.kind == Kind::medium)
        with(Medium{});
    else
        with(std::conditional_t<PLANES, ThinTriple, Thin>{});
}

struct Offsets {
    size_t at = 0;
    size_t take(size_t bytes)
    {
        const size_t o = at;
        at += (std::max<size_t>(bytes, 16) + 255) & ~size_t(255);
        return o;
    }
};

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
int planes(const CeProblem &p) { return p.type == ElemType::f32 ? 3 : 1; }
int64_t all_rows(const CeProblem &p) { return (int64_t)p.samples * p.rows; }

// x is copied where its rows are no whole steps (the copy's zeros are what ends
// the sums), w only where its rows cannot be read 16 bytes at a time.
void choose_packs(const CeProblem &p, bool *x, bool *w)
{
    *x = p.type == ElemType::f32 || p.dim % kCeStep || !aligned16(p.x);
    *w = p.type == ElemType::f32 || p.dim % 8 || !aligned16(p.w);
}

// Whether a forward pass in float32 multiplies x and w as they are: where the rows
// are one tile it is bound by w, which is then read once instead of copied into
// planes that are read (one row of 131072 x 4096: 396 us, by planes 2084; 128 rows
// 977 and 2038); with more rows the planes' products are the faster ones.
bool whole_float32(const CeProblem &p)
{
    return p.type == ElemType::f32 && p.rows <= 128 && p.dim % (kCeStep / 2) == 0 && aligned16(p.x) && aligned16(p.w);
}

// The copies that a pass needs, in one launch.
struct Packs {
    PackJobs jobs{};
    int n = 0;
    unsigned blocks = 0;
    void add(const void *in, uint16_t *out, int64_t samples, int rows, int rows_out, bool scaled)
    {
        PackJob &j = jobs.job[n++];
        j.in = in;
        j.out = out;
        j.n = samples * rows_out * jobs.dim_pad;
        j.rows = rows;
        j.rows_out = rows_out;
        j.scaled = scaled;
        j.blocks = blocks_for(j.n / 8, kBlock);
        blocks += j.blocks;
    }
    template <class IN> void launch(hipStream_t s) const
    {
        if (blocks)
            k_ce_pack<IN><<<dim3(blocks), dim3(kBlock), 0, s>>>(jobs);
    }
};

// The logits' scale in units of log 2; never 0, by which a class that is not
// there (an infinite logit) would become NaN.
float scale2_of(const CeProblem &p)
{
    const float s = p.scale * kLog2E;
    return std::abs(s) < FLT_MIN ? std::copysign(FLT_MIN, s) : s;
}

// Gradients whose parts wait to be added up.
template <class OUT> struct Joins {
    JoinJobs<OUT> jobs{};
    int n = 0;
    void add(const float *part, void *out, int64_t rows, int64_t split, int splits, const CeCoef *coef)
    {
        jobs.job[n++] = JoinJob{part, out, rows, split, splits, coef, blocks_for(rows * jobs.ld / 4, kBlock)};
    }
    void launch(hipStream_t s)
    {
        if (n)
            k_ce_join<OUT><<<dim3(jobs.job[0].blocks + (n > 1 ? jobs.job[1].blocks : 0)), dim3(kBlock), 0, s>>>(jobs);
        n = 0;
    }
};

Targets targets_of(const CeProblem &p) { return {p.target, p.target32, p.classes, p.ignore_index}; }

// x, w as operands with the features contiguous.
Operand features(const CeProblem &p, bool packed, const void *user, const uint16_t *copy, int64_t rows, int dim_pad)
{
    Operand o;
    o.base = packed ? copy : (const uint16_t *)user;
    o.ld = packed ? dim_pad : p.dim;
    o.sample = rows * o.ld;
    o.plane = p.samples * o.sample;
    o.rows = (int)rows;
    o.k = packed ? dim_pad : p.dim;
    return o;
}

template <class F> void by_type(ElemType t, F f)
{
    if (t == ElemType::f32)
        f(Bf16{}, std::true_type{}, float{});
    else if (t == ElemType::bf16)
        f(Bf16{}, std::false_type{}, Bf16{});
    else
        f(F16{}, std::false_type{}, F16{});
}

} // namespace

// The products in tiles of 128 x 128, 256 threads each: larger ones have half as
// many a result or fewer, those of 16 rows stand where there are no more, and a sum
// is cut into parts only where its tiles are few. The logits' gradient is cut into
// pieces far below the limit.
bool ce_launches_fit(const CeProblem &p)
{
    constexpr int64_t limit = ((int64_t)1 << 32) - 8 * kBlock; // every job of a launch ends in whole workgroups
    const int64_t rows = (int64_t)ceil_to(p.rows, 128) * p.samples, classes = (int64_t)ceil_to(p.classes, 128) * p.samples;
    const int64_t features = ceil_to(p.dim, 128), dim_pad = pad_to(p.dim, kCeStep);
    bool x, w;
    choose_packs(p, &x, &w);
    const int64_t copied = (x ? all_rows(p) : 0) + (w ? (int64_t)p.samples * p.classes : 0) +
                           p.samples * pad_to(p.rows, kCeStep);
    return rows * ceil_to(p.classes, 128) * 256 < limit && (rows + classes) * features * 256 < limit &&
           copied * dim_pad / 8 + all_rows(p) < limit && p.rows * pad_to(p.dim, 4) / 4 < limit;
}

// Threads of k_ce_rows a row: with few rows, as many as it takes to have the
// parts' loads in flight together (one row of 131072 classes, 4096 parts: 16
// threads 105 us, 256 threads 5.5 us), with many as few as let a workgroup read
// whole lines of each part.
static int row_threads(int64_t n) { return n >= 32768 ? 4 : n >= 256 ? 16 : kBlock; }

CeForwardPlan ce_plan_forward(const CeProblem &p)
{
    CeForwardPlan f{};
    f.whole_f32 = whole_float32(p);
    if (!f.whole_f32)
        choose_packs(p, &f.pack_x, &f.pack_w);
    f.dim_pad = (int)pad_to(p.dim, kCeStep);
    const Kind kind = f.whole_f32 && p.rows > 16 ? Kind::medium : choose(p.classes, p.rows, p.samples, true);
    f.parts = ceil_to(p.classes, tile_p(kind)) * waves_p(kind);
    const int64_t n = all_rows(p);
    Offsets o;
    f.x = o.take(f.pack_x ? n * f.dim_pad * 2 * planes(p) : 0);
    f.w = o.take(f.pack_w ? (int64_t)p.samples * p.classes * f.dim_pad * 2 * planes(p) : 0);
    f.part = o.take((int64_t)f.parts * n * sizeof(float2));
    f.picked = o.take(n * sizeof(float));
    f.sums = o.take(p.reduction == 0 ? 0 : blocks_for(n, kBlock / row_threads(n)) * sizeof(LossSum));
    f.ticket = o.take(sizeof(int));
    f.bytes = o.at;
    return f;
}

void ce_forward(const CeProblem &p, const CeForwardPlan &plan, uint8_t *ws, float *loss, CeRow *rows, float *total,
                hipStream_t s)
{
    const int64_t n = all_rows(p);
    auto *part = (float2 *)(ws + plan.part);
    auto *picked = (float *)(ws + plan.picked);
    auto *sums = (LossSum *)(ws + plan.sums);
    auto *ticket = (int *)(ws + plan.ticket);
    const Targets target = targets_of(p);
    auto *x = (uint16_t *)(ws + plan.x), *w = (uint16_t *)(ws + plan.w);
    const FinishStats finish{target, part, picked, ticket, scale2_of(p)};
    if (plan.whole_f32) {
        Product a{};
        a.p = features(p, false, p.w, nullptr, p.classes, 0);
        a.q = features(p, false, p.x, nullptr, p.rows, 0);
        for (Operand *o : {&a.p, &a.q}) { // in 16-bit elements
            o->ld *= 2;
            o->sample *= 2;
            o->k *= 2;
        }
        a.steps = a.p.k / kCeStep;
        a.samples = p.samples;
        a.splits = 1;
        if (p.rows <= 16)
            launch_shape<F32, false, Narrow>(a, p.classes, p.rows, finish, s);
        else
            launch_shape<F32, false, Medium>(a, p.classes, p.rows, finish, s);
    } else by_type(p.type, [&](auto elem, auto cut, auto io) {
        using ELEM = decltype(elem);
        using IO = decltype(io);
        Packs packs;
        packs.jobs.dim = p.dim;
        packs.jobs.dim_pad = plan.dim_pad;
        if (plan.pack_x)
            packs.add(p.x, x, p.samples, p.rows, p.rows, false);
        if (plan.pack_w)
            packs.add(p.w, w, p.samples, p.classes, p.classes, false);
        packs.launch<IO>(s);
        Product a{};
        a.p = features(p, plan.pack_w, p.w, w, p.classes, plan.dim_pad);
        a.q = features(p, plan.pack_x, p.x, x, p.rows, plan.dim_pad);
        a.steps = plan.dim_pad / kCeStep;
        a.samples = p.samples;
        a.splits = 1;
        launch_product<ELEM, decltype(cut)::value>(choose(p.classes, p.rows, p.samples, true), a, p.classes, p.rows,
                                                   finish, s);
    });
    const auto join = [&](auto threads) {
        constexpr int T = decltype(threads)::value;
        k_ce_rows<T><<<dim3(blocks_for(n, kBlock / T)), dim3(kBlock), 0, s>>>(
            part, plan.parts, picked, target, n, p.z_weight, p.reduction, loss, rows, sums, ticket, loss, total);
    };
    if (row_threads(n) == 4)
        join(std::integral_constant<int, 4>{});
    else if (row_threads(n) == 16)
        join(std::integral_constant<int, 16>{});
    else
        join(std::integral_constant<int, kBlock>{});
}

namespace {

// The piece of the logits' gradient that exists at a time: about what the 256 MB
// last-level cache keeps between the product that writes it and the two that
// read it. Smaller pieces are more launches, each with a tail (64, 128, 256, 512
// MB: 16 x 4096 x 16384 x 256 4.21, 3.72, 3.45, 3.56 ms before the gradients shared
// a launch; 128 and 256 MB now: 32 x 2048 x 2048 x 64 float32 676 and 689 us, one
// sample of 20000 x 20000 x 64 1895 and 1790).
constexpr int64_t kPieceBytes = (int64_t)256 << 20;
// A sample is cut along its classes, 256 at least; where its rows are too many for
// that (524288 in 16 bits, 262144 or 174762 in float32) along its rows as well, into
// pieces of about kCutClasses classes (600000 x 5000 x 256 bfloat16 9.8 ms, along the
// classes alone 16.2; 200000 x 3000 x 128 float32 5.9 and 7.4).
constexpr int64_t kLeastClasses = 256, kCutClasses = 2048;

// Whether the logits' gradient is stored in float32 as it is, two thirds of its
// planes: where the gradients' tile is ThinTriple.
bool whole_gradient(const CeProblem &p) { return p.type == ElemType::f32 && p.dim <= 64; }

// The gradients' launch of a whole piece.
Cut cut_of(const CeProblem &p, const CeBackwardPlan &b, bool want_x, bool want_w)
{
    return choose_grads(p.dim, b.piece_rows, b.piece_classes, b.piece_samples, ceil_to(b.piece_classes, kCeStep),
                        b.g_rows / kCeStep, planes(p), want_x, want_w);
}

} // namespace

// Lanes that read a row of float16 features, 16 bytes each, of a wave.
static int lanes_of(int dim)
{
    int lanes = 1;
    while (lanes < 64 && lanes * 8 < dim)
        lanes <<= 1;
    return lanes;
}

CeBackwardPlan ce_plan_backward(const CeProblem &p, bool want_x, bool want_w)
{
    CeBackwardPlan b{};
    choose_packs(p, &b.pack_x, &b.pack_w);
    b.dim_pad = (int)pad_to(p.dim, kCeStep);
    b.rows_pad = (int)pad_to(p.rows, kCeStep);
    b.whole_g = whole_gradient(p);
    const int64_t n = all_rows(p), size = 2 * planes(p), size_g = b.whole_g ? 4 : size;
    const auto bytes_of = [&](int64_t rows, int64_t classes) { return pad_to(rows, kCeStep) * pad_to(classes, kCeStep) * size_g; };
    b.piece_samples = 1;
    b.piece_rows = p.rows;
    b.piece_classes = p.classes;
    const int64_t whole = bytes_of(p.rows, p.classes); // of one sample
    if (whole <= kPieceBytes) {
        const int pieces = ceil_to(p.samples, kPieceBytes / whole); // of about as many samples each
        b.piece_samples = ceil_to(p.samples, pieces);
    } else {
        if (bytes_of(p.rows, std::min<int64_t>(p.classes, kLeastClasses)) > kPieceBytes) {
            const int64_t most = kPieceBytes / bytes_of(1, std::min<int64_t>(p.classes, kCutClasses)) * kCeStep / 256 * 256;
            b.piece_rows = (int)std::min<int64_t>(p.rows, pad_to(ceil_to(p.rows, ceil_to(p.rows, most)), 256));
        }
        if (bytes_of(b.piece_rows, p.classes) > kPieceBytes) {
            const int64_t most =
                std::max(kLeastClasses, kPieceBytes / (pad_to(b.piece_rows, kCeStep) * size_g) / 256 * 256);
            b.piece_classes = (int)std::min<int64_t>(p.classes, pad_to(ceil_to(p.classes, ceil_to(p.classes, most)), 256));
        }
    }
    b.g_rows = (int)pad_to(b.piece_rows, kCeStep);
    b.ld_g = (int)pad_to(b.piece_classes, kCeStep);
    // rows that lie a multiple of 2 KB apart share memory channels (16 x 4096 x
    // 16384 x 256: 3.42 ms, so 3.32; float32's three planes 0.89 and 0.90 ms)
    if (p.type != ElemType::f32 && b.ld_g % 1024 == 0)
        b.ld_g += 192;
    const Cut cut = cut_of(p, b, want_x, want_w);
    b.split_x = cut.split_x;
    b.split_w = cut.split_w;
    b.sum_x = b.split_x > 1 || b.piece_classes < p.classes;
    b.sum_w = b.split_w > 1 || b.piece_rows < p.rows;
    const int64_t ld = pad_to(p.dim, 4);
    Offsets o;
    b.x = o.take(b.pack_x ? n * b.dim_pad * size : 0);
    b.w = o.take(b.pack_w ? (int64_t)p.samples * p.classes * b.dim_pad * size : 0);
    b.coef = o.take(n * sizeof(CeCoef));
    const bool uneven = p.reduction == 0 || p.z_weight != 0.0f;
    b.size_lanes = uneven && want_w && p.type == ElemType::f16 ? lanes_of(p.dim) : 0;
    b.tops = uneven ? (int)std::min<int64_t>(512, blocks_for(n * std::max(b.size_lanes, 1), kBlock)) : 0;
    b.block_top = o.take(b.tops * sizeof(Largest));
    b.top = o.take(sizeof(CeTop));
    b.xs = o.take(want_w ? (int64_t)p.samples * b.rows_pad * b.dim_pad * size : 0);
    b.g = o.take((int64_t)b.piece_samples * b.g_rows * b.ld_g * size_g);
    // x's sums wait for all pieces of the classes, w's for a piece's rows alone
    const int64_t part_rows = b.piece_classes < p.classes ? p.rows : b.piece_rows;
    b.part_x = o.take(want_x && b.sum_x ? b.split_x * b.piece_samples * part_rows * ld * 4 : 0);
    b.part_w = o.take(want_w && b.sum_w ? (int64_t)b.split_w * b.piece_samples * b.piece_classes * ld * 4 : 0);
    b.bytes = o.at;
    // alone a gradient may be cut into more parts: room for both is room for either
    if (want_x && want_w)
        b.bytes = std::max({b.bytes, ce_plan_backward(p, true, false).bytes, ce_plan_backward(p, false, true).bytes});
    return b;
}

void ce_backward(const CeProblem &p, const CeBackwardPlan &plan, uint8_t *ws, const CeRow *rows, const float *total,
                 const float *grad_loss, void *grad_x, void *grad_w, hipStream_t s)
{
    const int64_t n = all_rows(p);
    auto *coef = (CeCoef *)(ws + plan.coef);
    auto *block_top = (Largest *)(ws + plan.block_top);
    auto *top = (CeTop *)(ws + plan.top);
    const Targets target = targets_of(p);
    const Upstream up{grad_loss, total, p.reduction, p.scale};
    auto *x = (uint16_t *)(ws + plan.x), *w = (uint16_t *)(ws + plan.w);
    auto *xs = (uint16_t *)(ws + plan.xs), *g = (uint16_t *)(ws + plan.g);
    auto *part_x = (float *)(ws + plan.part_x), *part_w = (float *)(ws + plan.part_w);
    const int64_t ld = pad_to(p.dim, 4);
    by_type(p.type, [&](auto elem, auto cut, auto io) {
        using ELEM = decltype(elem);
        using IO = decltype(io);
        constexpr bool PLANES = decltype(cut)::value;
        const float inv_unit = 1.0f / ELEM::kUnit;
        if (plan.tops && plan.size_lanes)
            k_ce_size<true><<<dim3(plan.tops), dim3(kBlock), 0, s>>>(rows, target, up, p.z_weight, n, (const uint16_t *)p.x,
                                                                     p.dim, plan.size_lanes, block_top);
        else if (plan.tops)
            k_ce_size<false><<<dim3(plan.tops), dim3(kBlock), 0, s>>>(rows, target, up, p.z_weight, n, nullptr, 0, 1,
                                                                      block_top);
        Packs packs;
        packs.jobs.dim = p.dim;
        packs.jobs.dim_pad = plan.dim_pad;
        packs.jobs.coefs = Coefs{rows, target, up, p.z_weight, ELEM::kUnit, block_top, plan.tops};
        packs.jobs.coef_rows = n;
        packs.jobs.coef = coef;
        packs.jobs.top = top;
        packs.blocks = packs.jobs.coef_blocks = blocks_for(n, kBlock);
        if (plan.pack_x)
            packs.add(p.x, x, p.samples, p.rows, p.rows, false);
        if (plan.pack_w)
            packs.add(p.w, w, p.samples, p.classes, p.classes, false);
        if (grad_w)
            packs.add(p.x, xs, p.samples, p.rows, plan.rows_pad, true);
        packs.launch<IO>(s);
        const Operand W = features(p, plan.pack_w, p.w, w, p.classes, plan.dim_pad);
        const Operand X = features(p, plan.pack_x, p.x, x, p.rows, plan.dim_pad);
        const Cut cut_grads = cut_of(p, plan, grad_x, grad_w);
        Joins<IO> joins;
        joins.jobs.cols = p.dim;
        joins.jobs.ld = (int)ld;
        joins.jobs.top = top;
        joins.jobs.inv_unit = inv_unit;
        // one piece after another: its samples from s0, classes from c0, rows from r0
        const auto piece = [&](int s0, int c0, int r0) {
            const int ns = std::min(plan.piece_samples, p.samples - s0); // more than one: with all classes and rows
            const int nc = std::min(plan.piece_classes, p.classes - c0), nc_pad = (int)pad_to(nc, kCeStep);
            const int nr = std::min(plan.piece_rows, p.rows - r0), nr_pad = (int)pad_to(nr, kCeStep);
            const int64_t row0 = (int64_t)s0 * p.rows + r0;
            const int64_t plane_g = (int64_t)plan.piece_samples * plan.g_rows * plan.ld_g;
            const TargetRest<IO> rest{target, (const uint16_t *)p.w + (int64_t)s0 * p.classes * p.dim, coef + row0, row0,
                                      nr, p.dim, inv_unit};
            { // the logits again, and their gradient
                Product a{};
                a.p = W;
                a.p.base += s0 * W.sample + (int64_t)c0 * W.ld;
                a.p.rows = nc;
                a.q = X;
                a.q.base += s0 * X.sample + r0 * X.ld;
                a.q.rows = nr;
                a.steps = plan.dim_pad / kCeStep;
                a.samples = ns;
                a.splits = 1;
                const auto product = [&](auto as) {
                    launch_product<ELEM, PLANES>(choose(nc, nr, ns, false), a, nc_pad, nr_pad,
                                                 FinishGrad<decltype(as)::value>{target, coef, row0, g, plane_g,
                                                                                 scale2_of(p), nr_pad, plan.ld_g, c0}, s);
                };
                if constexpr (!PLANES)
                    product(std::integral_constant<Stored, Stored::narrow>{});
                else if (plan.whole_g)
                    product(std::integral_constant<Stored, Stored::whole>{});
                else
                    product(std::integral_constant<Stored, Stored::planes>{});
            }
            Operand G;
            G.base = g;
            G.sample = (int64_t)nr_pad * plan.ld_g;
            G.plane = plane_g;
            G.ld = plan.ld_g;
            if (plan.whole_g) { // in 16-bit elements
                G.sample *= 2;
                G.ld *= 2;
            }
            GradJob<IO> jx{}, jw{};
            const bool cut_classes = nc < p.classes;
            const int64_t sample_x = (int64_t)nr * ld, split_x = cut_classes ? p.rows * ld : ns * sample_x;
            float *sum_x = part_x + (cut_classes ? r0 * ld : 0);
            void *to_x = (uint8_t *)grad_x + row0 * p.dim * elem_size(p.type);
            {
                Product &a = jx.a;
                a.p = W;
                a.p.base += s0 * W.sample + (int64_t)c0 * W.ld;
                a.p.rows = p.dim;
                a.p.k = nc;
                a.q = G;
                a.q.rows = nr;
                a.q.k = nc_pad;
                a.steps = nc_pad / kCeStep;
                a.samples = ns;
                a.splits = plan.split_x;
                jx.out.in_parts = plan.sum_x;
                jx.out.part = FinishPart{sum_x, split_x, sample_x, (int)ld, c0 > 0};
                jx.out.store = FinishStore<IO>{to_x, rest, coef + row0, top, inv_unit, (int64_t)p.rows * p.dim};
            }
            const int64_t sample_w = nc * ld, split_w = ns * sample_w, whole = (int64_t)p.classes * p.dim;
            void *to_w = (uint8_t *)grad_w + (s0 * whole + (int64_t)c0 * p.dim) * elem_size(p.type);
            {
                Product &a = jw.a;
                a.p.base = xs + ((int64_t)s0 * plan.rows_pad + r0) * plan.dim_pad;
                a.p.sample = (int64_t)plan.rows_pad * plan.dim_pad;
                a.p.plane = p.samples * a.p.sample;
                a.p.ld = plan.dim_pad;
                a.p.rows = p.dim;
                a.p.k = nr_pad;
                a.q = G;
                a.q.rows = nc;
                a.q.k = nr_pad;
                a.steps = nr_pad / kCeStep;
                a.samples = ns;
                a.splits = plan.split_w;
                jw.out.in_parts = plan.sum_w;
                jw.out.part = FinishPart{part_w, split_w, sample_w, (int)ld, r0 > 0};
                jw.out.store = FinishStore<IO>{to_w, rest, nullptr, top, inv_unit, whole};
            }
            launch_gradients<ELEM, PLANES>(cut_grads, jx, jw, grad_x, grad_w, s);
            // what is complete is joined while its parts are in the cache and before
            // the next piece writes over them
            joins.jobs.rest = rest;
            if (grad_w && plan.sum_w && r0 + nr == p.rows)
                joins.add(part_w, to_w, (int64_t)ns * nc, split_w, plan.split_w, nullptr);
            if (grad_x && plan.sum_x && c0 + nc == p.classes)
                joins.add(sum_x, to_x, (int64_t)ns * nr, split_x, plan.split_x, coef + row0);
            joins.launch(s);
        };
        for (int s0 = 0; s0 < p.samples; s0 += plan.piece_samples)
            for (int c0 = 0; c0 < p.classes; c0 += plan.piece_classes)
                for (int r0 = 0; r0 < p.rows; r0 += plan.piece_rows)
                    piece(s0, c0, r0);
    });
}

} // namespace apml
