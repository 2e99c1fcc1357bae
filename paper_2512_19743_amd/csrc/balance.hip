// Balance loss of a network with routed experts, per sample of T tokens and E
// experts, with p_t = softmax(logits_t) over the valid tokens (n of them), and
// the tokens that each expert was given:
//
//   P_e = (1 / n) sum_t p_te,   f_e = counts_e / sum counts
//   loss = E sum_e f_e P_e + z_weight (1 / n) sum_t lse_t^2
//   d loss / d logit_tj = (1 / n) p_tj (E f_j - sum_e E f_e p_te + 2 z_weight lse_t)
//
// Both directions read the logits once (the backward pass recomputes the
// softmax: storing it would cost a write and a read instead of one read) and
// are bound by that traffic. A token's row lies across `lanes` lanes of a wave,
// each with the same columns of every token, so that the sums P over the tokens
// stay in registers until a workgroup's chunk of tokens ends.
//
// Since sum_e p_te = 1, any number may be taken from all f: the backward pass has
// E (f_e - min f). Where the experts' shares are nearly equal the gradient is what is
// left of them, and it would be a difference of nearly equal numbers (8 experts all
// chosen, 6% of the slots dropped: 2e-5 off in float32, so 2e-7); d <= E f, so it
// is never further off than with f itself, and 0 where all shares are equal.
#include <algorithm>

#include "apml_internal.h"
#include "balance.h"
#include "device_common.h"

namespace apml {

namespace {

struct LoadF32 {
    using raw = float;
    static constexpr int wide = 4;
    static __device__ __forceinline__ float to(float v) { return v; }
    static __device__ __forceinline__ float from(float v) { return v; }
};
struct LoadBf16 {
    using raw = uint16_t;
    static constexpr int wide = 8;
    static __device__ __forceinline__ float to(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
    static __device__ __forceinline__ uint16_t from(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
};
struct LoadF16 {
    using raw = uint16_t;
    static constexpr int wide = 8;
    static __device__ __forceinline__ float to(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
    static __device__ __forceinline__ uint16_t from(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
};

template <class T, int VEC> struct alignas(sizeof(T) * VEC) Pack {
    T v[VEC];
};

// Butterfly over an aligned group of lanes, all of which end with the same bits.
template <class F> __device__ __forceinline__ float group_reduce(float v, int lanes, F f)
{
    const auto step = [&](auto k) {
        constexpr int K = decltype(k)::value;
        v = f(v, __builtin_bit_cast(float, partner<K>(__builtin_bit_cast(int, v))));
    };
    if (lanes > 1)
        step(std::integral_constant<int, 0>{});
    if (lanes > 2)
        step(std::integral_constant<int, 1>{});
    if (lanes > 4)
        step(std::integral_constant<int, 2>{});
    if (lanes > 8)
        step(std::integral_constant<int, 3>{});
    if (lanes > 16)
        step(std::integral_constant<int, 4>{});
    if (lanes > 32)
        step(std::integral_constant<int, 5>{});
    return v;
}
__device__ __forceinline__ float group_max(float v, int lanes)
{
    return group_reduce(v, lanes, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float group_add(float v, int lanes)
{
    return group_reduce(v, lanes, [](float a, float b) { return a + b; });
}

// Columns of a lane: VEC neighbours at (i * lanes + lane) * VEC, i < NV.
// A missing column reads as -inf.
template <class L, int VEC, int NV>
__device__ __forceinline__ void load_row(const typename L::raw *row, int lane, int lanes, int E, float (&v)[NV * VEC])
{
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * lanes + lane) * VEC;
        if (c < E) { // VEC > 1 only where E is a multiple of it
            const auto p = *(const Pack<typename L::raw, VEC> *)(row + c);
#pragma unroll
            for (int u = 0; u < VEC; ++u)
                v[i * VEC + u] = L::to(p.v[u]);
        } else {
#pragma unroll
            for (int u = 0; u < VEC; ++u)
                v[i * VEC + u] = -kInf;
        }
    }
}

// Rows that cannot be read 16 bytes at a time pass through shared memory: their
// tokens lie one after another, so a tile of them is read in whole 16-byte words
// wherever it starts (13 x 7001 tokens of 161 experts in half precision, backward:
// 31 us, element by element 42).
// An element keeps its place within its word; returns the first one's.
template <class R> __device__ __forceinline__ R *tile_in(R *lds, const R *src, int n)
{
    constexpr int W = 16 / sizeof(R);
    const int shift = (int)(((uintptr_t)src & 15) / sizeof(R));
    const int head = min(n, (W - shift) % W), words = (n - head) / W;
    R *to = lds + shift;
    for (int i = threadIdx.x; i < words; i += kBlock)
        *(Pack<R, W> *)(to + head + i * W) = *(const Pack<R, W> *)(src + head + i * W);
    const int tail = head + words * W;
    if ((int)threadIdx.x < head)
        to[threadIdx.x] = src[threadIdx.x];
    if ((int)threadIdx.x < n - tail)
        to[tail + threadIdx.x] = src[tail + threadIdx.x];
    return to;
}
template <class R> __device__ __forceinline__ void tile_out(R *dst, const R *from, int n)
{
    constexpr int W = 16 / sizeof(R);
    if ((((uintptr_t)dst ^ (uintptr_t)(__attribute__((address_space(3))) const R *)from) & 15) != 0) {
        for (int i = threadIdx.x; i < n; i += kBlock)
            dst[i] = from[i];
        return;
    }
    const int shift = (int)(((uintptr_t)dst & 15) / sizeof(R));
    const int head = min(n, (W - shift) % W), words = (n - head) / W;
    for (int i = threadIdx.x; i < words; i += kBlock)
        *(Pack<R, W> *)(dst + head + i * W) = *(const Pack<R, W> *)(from + head + i * W);
    const int tail = head + words * W;
    if ((int)threadIdx.x < head)
        dst[threadIdx.x] = from[threadIdx.x];
    if ((int)threadIdx.x < n - tail)
        dst[tail + threadIdx.x] = from[tail + threadIdx.x];
}

// v becomes exp(v - max); returns the log-sum-exp, and 1 / sum in *inv (0 for a
// row of -inf: it has no softmax and adds nothing). The exponential is that of base 2
// of the argument times log2 e, whose rounding moves a probability of e^-k by k 2^-24
// of itself.
template <int N> __device__ __forceinline__ float exp_row(float (&v)[N], int lanes, float *inv)
{
    float m = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i)
        m = fmaxf(m, v[i]);
    m = group_max(m, lanes);
    const float base = m == -kInf ? 0.0f : m;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = __expf(v[i] - base);
        s += v[i];
    }
    s = group_add(s, lanes);
    *inv = s == 0.0f ? 0.0f : 1.0f / s;
    return s == 0.0f ? 0.0f : base + __logf(s);
}

template <bool I32> __device__ __forceinline__ int64_t index_at(const void *index, int64_t i)
{
    return I32 ? (int64_t)((const int32_t *)index)[i] : ((const int64_t *)index)[i];
}

// The chosen experts of tokens [t0, t1) of a sample into an LDS histogram.
template <bool I32>
__device__ __forceinline__ void count_chunk(const void *index, const uint8_t *valid, int64_t token0, int tokens, int chosen,
                                            int E, int *hist, int threads)
{
    const int n = tokens * chosen;
    for (int i = threadIdx.x; i < n; i += threads) {
        const int64_t e = index_at<I32>(index, token0 * chosen + i);
        if (e >= 0 && e < E && (!valid || valid[token0 + i / chosen]))
            atomicAdd(&hist[(int)e], 1);
    }
}

struct ChunkSum {
    float z; // sum of lse^2
    int n;   // valid tokens
};

struct BalanceArgs {
    const void *logits, *index;
    const uint8_t *valid;
    int tokens, E, chosen, chunk, chunks, lanes;
    int tile;      // tokens that pass through shared memory at a time
    float z_weight;
    float *p;      // [samples][chunks][E]
    int32_t *count;
    ChunkSum *z;   // [samples][chunks]
    int *ticket;   // cleared for k_balance_join
};

// Tokens that a lane group adds up in float32 before its sums go into the chunk's, in
// double precision: equal addends, whose roundings all go one way, are off by half
// as many half steps at most (524288 equal tokens of 2 experts, 4096 a group, in one
// float32 sum: 5e-5 off). Both took the same time where a chunk is one run (16 x 8192
// x 64: 13.2 us).
constexpr int kRunTokens = 128;

// A chunk's sums of the probabilities, its tokens per expert and its sum of lse^2.
// Bound by the latency of few rows a lane group (16 x 8192 tokens of 64 experts in
// bfloat16, 17 MB: 14 us) and, for rows of odd length, by the exponentials.
template <class L, int VEC, int NV>
__global__ __launch_bounds__(kBlock) void k_balance_chunks(BalanceArgs a, bool index32)
{
    extern __shared__ __attribute__((aligned(16))) double sm[]; // [E] sums, then [E] counts
    __shared__ double sz[kBlock / 64];
    __shared__ int sn[kBlock / 64];
    int *hist = (int *)(sm + a.E);
    const int sample = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const int t0 = chunk * a.chunk, t1 = min(t0 + a.chunk, a.tokens);
    const int lane = threadIdx.x & (a.lanes - 1), group = threadIdx.x / a.lanes, groups = kBlock / a.lanes;
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *a.ticket = 0;
    for (int e = threadIdx.x; e < a.E; e += kBlock) {
        sm[e] = 0.0;
        hist[e] = 0;
    }
    __syncthreads();
    const int64_t row0 = (int64_t)sample * a.tokens;
    if (a.index) {
        if (index32)
            count_chunk<true>(a.index, a.valid, row0 + t0, t1 - t0, a.chosen, a.E, hist, kBlock);
        else
            count_chunk<false>(a.index, a.valid, row0 + t0, t1 - t0, a.chosen, a.E, hist, kBlock);
    }
    float acc[NV * VEC], z = 0.0f;
    double zs = 0.0;
    int n = 0;
    const int wave = threadIdx.x >> 6, in_wave = threadIdx.x & 63;
    const auto add = [&](float (&v)[NV * VEC]) {
        float inv;
        const float lse = exp_row(v, a.lanes, &inv);
#pragma unroll
        for (int i = 0; i < NV * VEC; ++i)
            acc[i] = __builtin_fmaf(v[i], inv, acc[i]);
        z = __builtin_fmaf(lse, lse, z);
        ++n;
    };
    for (int r0 = t0; r0 < t1; r0 += groups * kRunTokens) {
        const int r1 = min(r0 + groups * kRunTokens, t1);
#pragma unroll
        for (int i = 0; i < NV * VEC; ++i)
            acc[i] = 0.0f;
        if constexpr (VEC > 1) {
            for (int t = r0 + group; t < r1; t += 2 * groups) { // two rows' loads in flight
                const int64_t r = row0 + t, q = r + groups;
                const bool two = t + groups < r1;
                const bool vr = !a.valid || a.valid[r], vq = two && (!a.valid || a.valid[q]);
                float v[NV * VEC], w[NV * VEC];
                load_row<L, VEC, NV>((const typename L::raw *)a.logits + r * a.E, lane, a.lanes, a.E, v);
                load_row<L, VEC, NV>((const typename L::raw *)a.logits + (two ? q : r) * a.E, lane, a.lanes, a.E, w);
                if (vr)
                    add(v);
                if (vq)
                    add(w);
            }
        } else {
            using R = typename L::raw;
            R *lds = (R *)((float *)sm + ((3 * a.E + 3) & ~3));
            for (int b = r0; b < r1; b += a.tile) {
                const int n_tok = min(a.tile, r1 - b);
                __syncthreads();
                const R *rows = tile_in(lds, (const R *)a.logits + (row0 + b) * a.E, n_tok * a.E);
                __syncthreads();
                for (int t = group; t < n_tok; t += groups) {
                    if (a.valid && !a.valid[row0 + b + t])
                        continue;
                    float v[NV * VEC];
                    load_row<L, VEC, NV>(rows + t * a.E, lane, a.lanes, a.E, v);
                    add(v);
                }
            }
        }
        // the groups of a wave, then the waves one after another: a fixed order
        for (int o = a.lanes; o < 64; o <<= 1) {
#pragma unroll
            for (int i = 0; i < NV * VEC; ++i)
                acc[i] += __shfl_xor(acc[i], o);
        }
        for (int w = 0; w < kBlock / 64; ++w) {
            if (wave == w && in_wave < a.lanes) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int u = 0; u < VEC; ++u) {
                        const int c = (i * a.lanes + lane) * VEC + u;
                        if (c < a.E)
                            sm[c] += (double)acc[i * VEC + u];
                    }
            }
            __syncthreads();
        }
        zs += (double)z;
        z = 0.0f;
    }
    for (int o = a.lanes; o < 64; o <<= 1) {
        zs += __shfl_xor(zs, o);
        n += __shfl_xor(n, o);
    }
    if (in_wave == 0) {
        sz[wave] = zs;
        sn[wave] = n;
    }
    __syncthreads();
    const int64_t at = (int64_t)blockIdx.x * a.E;
    for (int e = threadIdx.x; e < a.E; e += kBlock) {
        a.p[at + e] = (float)sm[e];
        if (a.index)
            a.count[at + e] = hist[e];
    }
    if (threadIdx.x == 0) {
        for (int w = 1; w < kBlock / 64; ++w) {
            zs += sz[w];
            n += sn[w];
        }
        a.z[blockIdx.x] = ChunkSum{(float)zs, n};
    }
}

// A chunk's share of an expert.
struct Share {
    float p;
    int count;
};

// Joins a sample's chunks in double precision: one workgroup a sample (64 chunks
// of 64 experts: 9 us; one chunk of 8 experts 8 us, most of it a thread's 127 sums).
__global__ __launch_bounds__(1024) void k_balance_join(BalanceArgs a, int64_t *counts, float *loss, float *state,
                                                       int reduction, float *per, int *ticket)
{
    __shared__ double ssum[3][16]; // per wave
    __shared__ long long smin[16], least;
    __shared__ double total[3];
    __shared__ double sp[1024];
    __shared__ long long sc[1024];
    __shared__ bool is_last;
    const int sample = blockIdx.x;
    const int64_t base = (int64_t)sample * a.chunks;
    // 1024 / width threads an expert, each with every so-manieth chunk
    int width = 1;
    while (width < a.E)
        width <<= 1;
    const int e = threadIdx.x & (width - 1), k0 = threadIdx.x / width, step = 1024 / width;
    double p = 0.0;
    long long c = 0;
    if (e < a.E)
        strided<8>(
            k0, a.chunks, step,
            [&](int k) {
                return Share{a.p[(base + k) * a.E + e], a.index ? a.count[(base + k) * a.E + e] : 0};
            },
            [&](Share v, int) {
                p += (double)v.p;
                c += v.count;
            });
    sp[threadIdx.x] = p;
    sc[threadIdx.x] = c;
    double z = 0.0, n = 0.0;
    for (int k = threadIdx.x; k < a.chunks; k += 1024) {
        const ChunkSum v = a.z[base + k];
        z += (double)v.z;
        n += (double)v.n;
    }
    __syncthreads();
    const bool mine = (int)threadIdx.x < a.E;
    if (mine) {
        for (int k = 1; k < step; ++k) {
            p += sp[k * width + threadIdx.x];
            c += sc[k * width + threadIdx.x];
        }
        if (a.index)
            counts[(int64_t)sample * a.E + threadIdx.x] = c;
        else
            c = counts[(int64_t)sample * a.E + threadIdx.x];
    } else {
        p = 0.0;
        c = 0;
    }
    const auto reduce = [&](double v, int which) {
        v = wave_sum(v);
        if (lane_id() == 0)
            ssum[which][threadIdx.x >> 6] = v;
    };
    long long lowest = mine ? c : INT64_MAX;
    for (int o = 32; o > 0; o >>= 1)
        lowest = min(lowest, __shfl_xor(lowest, o));
    if (lane_id() == 0)
        smin[threadIdx.x >> 6] = lowest;
    reduce((double)c, 0);
    reduce(z, 1);
    reduce(n, 2);
    __syncthreads();
    if (threadIdx.x < 3) {
        double v = 0.0;
        for (int w = 0; w < 16; ++w)
            v += ssum[threadIdx.x][w];
        total[threadIdx.x] = v;
    } else if (threadIdx.x == 64) { // another wave
        for (int w = 0; w < 16; ++w)
            lowest = min(lowest, smin[w]);
        least = lowest;
    }
    __syncthreads();
    const double unit = (double)a.E / fmax(total[0], 1.0), load = unit * (double)c, inv_n = 1.0 / fmax(total[2], 1.0);
    if (mine && state)
        state[(int64_t)sample * (a.E + 1) + threadIdx.x] = (float)(unit * (double)(c - least));
    const double zz = total[1];
    __syncthreads();
    reduce(load * p, 0);
    __syncthreads();
    if (threadIdx.x == 0) {
        double v = 0.0;
        for (int w = 0; w < 16; ++w)
            v += ssum[0][w];
        v *= inv_n;
        if (a.z_weight != 0.0f)
            v += (double)a.z_weight * zz * inv_n;
        if (state)
            state[(int64_t)sample * (a.E + 1) + a.E] = (float)inv_n;
        if (reduction == 0 || gridDim.x == 1) {
            loss[sample] = (float)v;
        } else {
            // device-scope accesses go past the XCDs' own L2s: the wait is all
            // the order that the ticket needs
            __hip_atomic_store(&per[sample], (float)v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            is_last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
        }
    }
    if (reduction == 0 || gridDim.x == 1)
        return;
    __syncthreads();
    if (!is_last || threadIdx.x >= 64)
        return;
    double v = 0.0; // the samples in their order, by the last workgroup to end
    for (int i = threadIdx.x; i < (int)gridDim.x; i += 64)
        v += (double)__hip_atomic_load(&per[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    v = wave_sum(v);
    if (threadIdx.x == 0)
        loss[0] = (float)(reduction == 2 ? v / (double)gridDim.x : v);
}

// The logits' gradient, with the softmax computed again (16 x 8192 x 64 bfloat16,
// 34 MB read and written: 13 us).
template <class L, int VEC, int NV>
__global__ __launch_bounds__(kBlock) void k_balance_grad(BalanceArgs a, const float *state, const float *grad_loss,
                                                         int per_sample, float factor, void *out)
{
    const int sample = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const int t0 = chunk * a.chunk, t1 = min(t0 + a.chunk, a.tokens);
    const int lane = threadIdx.x & (a.lanes - 1), group = threadIdx.x / a.lanes, groups = kBlock / a.lanes;
    const float *load = state + (int64_t)sample * (a.E + 1);
    const float g = grad_loss[per_sample ? sample : 0] * factor * load[a.E];
    float f[NV * VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int u = 0; u < VEC; ++u) {
            const int c = (i * a.lanes + lane) * VEC + u;
            f[i * VEC + u] = c < a.E ? load[c] : 0.0f;
        }
    const int64_t row0 = (int64_t)sample * a.tokens;
    const auto finish = [&](float (&v)[NV * VEC], bool valid, typename L::raw *to) {
        if (valid) {
            float inv, dot = 0.0f;
            const float lse = exp_row(v, a.lanes, &inv);
#pragma unroll
            for (int i = 0; i < NV * VEC; ++i)
                dot = __builtin_fmaf(v[i], f[i], dot);
            dot = group_add(dot, a.lanes) * inv;
            const float shift = (a.z_weight != 0.0f ? 2.0f * a.z_weight * lse : 0.0f) - dot;
#pragma unroll
            for (int i = 0; i < NV * VEC; ++i)
                v[i] = g * (v[i] * inv) * (f[i] + shift);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * a.lanes + lane) * VEC;
            if (c < a.E) {
                Pack<typename L::raw, VEC> p;
#pragma unroll
                for (int u = 0; u < VEC; ++u)
                    p.v[u] = L::from(valid ? v[i * VEC + u] : 0.0f);
                *(Pack<typename L::raw, VEC> *)(to + c) = p;
            }
        }
    };
    if constexpr (VEC > 1) {
        for (int t = t0 + group; t < t1; t += 2 * groups) { // two rows' loads in flight
            const int64_t r = row0 + t, q = r + groups;
            const bool two = t + groups < t1;
            const bool vr = !a.valid || a.valid[r], vq = two && (!a.valid || a.valid[q]);
            float v[NV * VEC], w[NV * VEC];
            load_row<L, VEC, NV>((const typename L::raw *)a.logits + r * a.E, lane, a.lanes, a.E, v);
            load_row<L, VEC, NV>((const typename L::raw *)a.logits + (two ? q : r) * a.E, lane, a.lanes, a.E, w);
            finish(v, vr, (typename L::raw *)out + r * a.E);
            if (two)
                finish(w, vq, (typename L::raw *)out + q * a.E);
        }
    } else {
        extern __shared__ __attribute__((aligned(16))) double sm[];
        using R = typename L::raw;
        R *lds = (R *)sm;
        for (int b = t0; b < t1; b += a.tile) {
            const int n_tok = min(a.tile, t1 - b);
            const int64_t at = (row0 + b) * a.E;
            __syncthreads();
            R *rows = tile_in(lds, (const R *)a.logits + at, n_tok * a.E);
            __syncthreads();
            for (int t = group; t < n_tok; t += groups) {
                float v[NV * VEC];
                load_row<L, VEC, NV>(rows + t * a.E, lane, a.lanes, a.E, v);
                finish(v, !a.valid || a.valid[row0 + b + t], rows + t * a.E);
            }
            __syncthreads();
            tile_out((R *)out + at, rows, n_tok * a.E);
        }
    }
}

__global__ __launch_bounds__(kBlock) void k_counts_clear(unsigned long long *counts, int64_t n)
{
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i < n)
        counts[i] = 0;
}

// Integer sums: the order of the atomics does not show. Bound by the read of the
// indices (16.8 million int64, 134 MB: 29 us, 4.6 TB/s).
template <bool I32>
__global__ __launch_bounds__(kBlock) void k_counts(BalanceArgs a, unsigned long long *counts)
{
    __shared__ int hist[kMaxExperts];
    const int sample = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const int t0 = chunk * a.chunk, t1 = min(t0 + a.chunk, a.tokens);
    for (int e = threadIdx.x; e < a.E; e += kBlock)
        hist[e] = 0;
    __syncthreads();
    count_chunk<I32>(a.index, a.valid, (int64_t)sample * a.tokens + t0, t1 - t0, a.chosen, a.E, hist, kBlock);
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kBlock) {
        unsigned long long *to = &counts[(int64_t)sample * a.E + e];
        if (a.chunks == 1)
            *to = (unsigned long long)hist[e];
        else if (hist[e])
            atomicAdd(to, (unsigned long long)hist[e]);
    }
}

// Lanes of a token's row, and whether its columns are read 16 bytes at a time.
struct RowShape {
    int vec, nv, lanes;
};
RowShape row_shape(const BalanceProblem &p, const void *grad)
{
    const int wide = p.type == ElemType::f32 ? 4 : 8;
    RowShape r{1, 1, 1};
    if (p.experts % wide == 0 && ((uintptr_t)p.logits & 15) == 0 && ((uintptr_t)grad & 15) == 0)
        r.vec = wide;
    // 16 lanes, whose exchanges need no shared memory, take up to 4 packs each
    // (16 single columns); more lanes what is left
    const int packs = (p.experts + r.vec - 1) / r.vec;
    const int most = r.vec > 1 ? 4 : 16;
    r.nv = packs <= 16 ? 1 : packs <= 64 || r.vec > 1 ? 4 : most;
    while (r.lanes * r.nv < packs)
        r.lanes <<= 1;
    return r;
}

template <class F> void by_shape(ElemType t, const RowShape &r, F f)
{
    const auto with = [&](auto l) {
        using L = decltype(l);
        if (r.vec > 1 && r.nv == 4)
            f(l, std::integral_constant<int, L::wide>{}, std::integral_constant<int, 4>{});
        else if (r.vec > 1)
            f(l, std::integral_constant<int, L::wide>{}, std::integral_constant<int, 1>{});
        else if (r.nv == 16)
            f(l, std::integral_constant<int, 1>{}, std::integral_constant<int, 16>{});
        else if (r.nv == 4)
            f(l, std::integral_constant<int, 1>{}, std::integral_constant<int, 4>{});
        else
            f(l, std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{});
    };
    if (t == ElemType::f32)
        with(LoadF32{});
    else if (t == ElemType::bf16)
        with(LoadBf16{});
    else
        with(LoadF16{});
}

// Chunks of a sample's tokens: about `blocks` workgroups in all, each with at
// least `least` tokens.
void cut_tokens(const BalanceProblem &p, int64_t blocks, int least, int *chunk, int *chunks)
{
    const int64_t per = std::max<int64_t>(1, blocks / p.samples);
    *chunk = (int)std::max<int64_t>(least, (p.tokens + per - 1) / per);
    *chunks = (p.tokens + *chunk - 1) / *chunk;
}

// Tokens that pass through shared memory at a time: 16 KB of them, at least one a
// lane group.
int tile_tokens(const BalanceProblem &p, const RowShape &r)
{
    const int groups = kBlock / r.lanes, row = p.experts * (int)elem_size(p.type);
    return groups * std::max(1, 16384 / (row * groups));
}
size_t tile_bytes(const BalanceProblem &p, const RowShape &r)
{
    return r.vec > 1 ? 0 : (size_t)tile_tokens(p, r) * p.experts * elem_size(p.type) + 32;
}

// A few tokens a lane group of a workgroup, whose size grows with the experts.
int least_tokens(const BalanceProblem &p) { return std::min(512, std::max(16, 8192 / p.experts)); }

BalanceArgs args_of(const BalanceProblem &p)
{
    BalanceArgs a{};
    a.logits = p.logits;
    a.index = p.index;
    a.valid = p.valid;
    a.tokens = p.tokens;
    a.E = p.experts;
    a.chosen = p.chosen;
    a.z_weight = p.z_weight;
    return a;
}

} // namespace

BalancePlan balance_plan(const BalanceProblem &p)
{
    BalancePlan b{};
    cut_tokens(p, 1024, least_tokens(p), &b.tokens, &b.chunks);
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t o = at;
        at += (std::max<size_t>(bytes, 16) + 255) & ~size_t(255);
        return o;
    };
    const size_t parts = (size_t)p.samples * b.chunks;
    b.p = take(parts * p.experts * sizeof(float));
    b.count = take(parts * p.experts * sizeof(int32_t));
    b.z = take(parts * sizeof(ChunkSum));
    b.loss = take(p.samples * sizeof(float));
    b.ticket = take(sizeof(int));
    b.bytes = at;
    return b;
}

void balance_forward(const BalanceProblem &p, const BalancePlan &plan, uint8_t *ws, int64_t *counts, float *loss,
                     float *state, hipStream_t s)
{
    const RowShape r = row_shape(p, nullptr);
    BalanceArgs a = args_of(p);
    a.chunk = plan.tokens;
    a.chunks = plan.chunks;
    a.lanes = r.lanes;
    a.tile = tile_tokens(p, r);
    a.p = (float *)(ws + plan.p);
    a.count = (int32_t *)(ws + plan.count);
    a.z = (ChunkSum *)(ws + plan.z);
    a.ticket = (int *)(ws + plan.ticket);
    by_shape(p.type, r, [&](auto l, auto vec, auto nv) {
        k_balance_chunks<decltype(l), decltype(vec)::value, decltype(nv)::value>
            <<<dim3((unsigned)(p.samples * a.chunks)), dim3(kBlock),
               ((3 * p.experts + 3) & ~3) * sizeof(float) + tile_bytes(p, r), s>>>(a, p.index32);
    });
    k_balance_join<<<dim3(p.samples), dim3(1024), 0, s>>>(a, counts, loss, state, p.reduction, (float *)(ws + plan.loss),
                                                         a.ticket);
}

void balance_backward(const BalanceProblem &p, const float *state, const float *grad_loss, void *grad, hipStream_t s)
{
    const RowShape r = row_shape(p, grad);
    BalanceArgs a = args_of(p);
    a.lanes = r.lanes;
    a.tile = tile_tokens(p, r);
    cut_tokens(p, 4096, least_tokens(p) / 2, &a.chunk, &a.chunks);
    by_shape(p.type, r, [&](auto l, auto vec, auto nv) {
        k_balance_grad<decltype(l), decltype(vec)::value, decltype(nv)::value>
            <<<dim3((unsigned)(p.samples * a.chunks)), dim3(kBlock), tile_bytes(p, r), s>>>(
                a, state, grad_loss, p.reduction == 0, p.reduction == 2 ? 1.0f / (float)p.samples : 1.0f, grad);
    });
}

void expert_counts(const BalanceProblem &p, int64_t *counts, hipStream_t s)
{
    BalanceArgs a = args_of(p);
    cut_tokens(p, 2048, std::max(1, 2048 / p.chosen), &a.chunk, &a.chunks);
    const int64_t n = (int64_t)p.samples * p.experts;
    auto *to = (unsigned long long *)counts;
    if (a.chunks > 1)
        k_counts_clear<<<dim3(blocks_for(n, kBlock)), dim3(kBlock), 0, s>>>(to, n);
    if (p.index32)
        k_counts<true><<<dim3((unsigned)(p.samples * a.chunks)), dim3(kBlock), 0, s>>>(a, to);
    else
        k_counts<false><<<dim3((unsigned)(p.samples * a.chunks)), dim3(kBlock), 0, s>>>(a, to);
}

} // namespace apml
