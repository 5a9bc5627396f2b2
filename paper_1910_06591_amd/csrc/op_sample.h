// Sampling with temperature, top-k, top-p and min-p from one given uniform a row.
//
// The choices of a row are ordered by (logit descending, index ascending); every filter keeps a prefix of that order.
// An element's place in it is a 64-bit key, the logit's bits in an order that integers have, then the inverted index:
// larger key = earlier.  Masses exp((x - max) / T) are computed in 64 bits and added as 64-bit integers in units of
// 2^-shift of the largest: a sum's value does not depend on the order of its terms, so neither does a choice.
#pragma once
#include "op_common.h"

namespace seedinf {

struct SampleArgs {
    const void* logits; int64_t stride;          // [rows, choices], elements between rows
    const float* uniforms;                       // [rows]
    const float* temperature;                    // [rows] or nullptr (1); a row's value <= 0 or NaN: greedy
    const int32_t* top_k;                        // [rows] or nullptr; <= 0 or >= choices: off
    const float* top_p;                          // [rows] or nullptr; >= 1 or NaN: off
    const float* min_p;                          // [rows] or nullptr; <= 0 or NaN: off
    int32_t* token; float* logprob;              // logprob may be nullptr
    int rows, V;
    int shift;                                   // V * 2^shift < 2^63
};

// NaN never wins, and the two zeros are one value.
__device__ __forceinline__ float sample_clean(float x) { return x != x ? -INFINITY : x + 0.0f; }
__device__ __forceinline__ uint32_t sample_order(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t sample_key(float x, int i) { return (uint64_t)sample_order(x) << 32 | (uint32_t)~i; }

__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int off)
{
    const uint32_t lo = __shfl_xor((int)(uint32_t)v, off, 64), hi = __shfl_xor((int)(uint32_t)(v >> 32), off, 64);
    return (uint64_t)hi << 32 | lo;
}

struct SampleRow {
    float top;                   // the largest logit
    double inv_t;
    double unit;                 // 2^shift
    // the equal of an infinite largest logit has mass 1, a masked choice none at any temperature
    __device__ __forceinline__ double exponent(float x) const { return x == top ? 0.0 : (x == -INFINITY ? -INFINITY : ((double)x - (double)top) * inv_t); }
    __device__ __forceinline__ double mass(float x) const { return exp(exponent(x)); }
    __device__ __forceinline__ uint64_t units(double m) const { return (uint64_t)(m * unit + 0.5); }
};

constexpr int SAMPLE_THREADS = 256;
constexpr int SAMPLE_BITS = 11, SAMPLE_BINS = 1 << SAMPLE_BITS;

// Radix search for one place of the order, from the largest key down, 11 bits of the key a pass: the first element
// at which the running count reaches `count` (mass = false), or the running mass reaches (strict = false) or exceeds
// (strict = true) `limit`.  Returns its key.  There has to be one.
template <class T>
__device__ uint64_t sample_find(const T* x, const SampleArgs& p, const SampleRow& row, bool mass, bool strict, uint64_t count, double limit,
                                uint64_t* hist, uint64_t* share)
{
    const int tid = threadIdx.x;
    uint64_t prefix = 0, before = 0;
    int low = 64;                                            // key bits below `low` are not yet known
    while (low > 0) {
        const int w = low < SAMPLE_BITS ? low : SAMPLE_BITS, at = low - w;
        for (int i = tid; i < SAMPLE_BINS; i += SAMPLE_THREADS) hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < p.V; i += SAMPLE_THREADS) {
            const float f = sample_clean((float)x[i]);
            const uint64_t key = sample_key(f, i);
            if (low < 64 && (key >> low) != prefix) continue;
            const uint64_t add = mass ? row.units(row.mass(f)) : 1;
            if (add) atomicAdd((unsigned long long*)&hist[(key >> at) & ((1u << w) - 1)], (unsigned long long)add);
        }
        __syncthreads();
        if (tid == 0) {                                      // bins from the top
            uint64_t run = before;
            int bin = (1 << w) - 1;
            for (; bin > 0; --bin) {
                const uint64_t next = run + hist[bin];
                if (mass ? (strict ? (double)next > limit : (double)next >= limit) && hist[bin] : next >= count) break;
                run = next;
            }
            share[0] = (uint64_t)bin;
            share[1] = run;
        }
        __syncthreads();
        prefix = prefix << w | share[0];
        before = share[1];
        low = at;
    }
    return prefix;
}

__device__ __forceinline__ uint64_t sample_block_sum(uint64_t v, uint64_t* scratch)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += shfl_xor64(v, off);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    uint64_t s = 0;
    for (int i = 0; i < SAMPLE_THREADS / 64; ++i) s += scratch[i];
    return s;
}

// One workgroup per row; every question about the order is a radix search over the row.
template <class T>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(SampleArgs p)
{
    __shared__ uint64_t hist[SAMPLE_BINS];
    __shared__ uint64_t scratch[SAMPLE_THREADS / 64];
    __shared__ uint64_t share[2];
    const int r = blockIdx.x, tid = threadIdx.x;
    const T* x = (const T*)p.logits + (int64_t)r * p.stride;
    // the first of the order
    uint64_t best = 0;
    for (int i = tid; i < p.V; i += SAMPLE_THREADS) {
        const uint64_t key = sample_key(sample_clean((float)x[i]), i);
        best = key > best ? key : best;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) { const uint64_t o = shfl_xor64(best, off); best = o > best ? o : best; }
    if ((tid & 63) == 0) scratch[tid >> 6] = best;
    __syncthreads();
    for (int i = 0; i < SAMPLE_THREADS / 64; ++i) best = scratch[i] > best ? scratch[i] : best;
    const int first = (int)~(uint32_t)best;
    SampleRow row;
    row.top = sample_clean((float)x[first]);
    if (row.top == -INFINITY) {
        if (tid == 0) { p.token[r] = -1; if (p.logprob) p.logprob[r] = -INFINITY; }
        return;
    }
    const float temp = p.temperature ? p.temperature[r] : 1.0f;
    if (!(temp > 0.0f)) {
        if (tid == 0) { p.token[r] = first; if (p.logprob) p.logprob[r] = 0.0f; }
        return;
    }
    row.inv_t = 1.0 / (double)temp;
    row.unit = (double)(1ull << p.shift);
    // the last kept key
    uint64_t last = 0;
    const int k = p.top_k ? p.top_k[r] : 0;
    if (k > 0 && k < p.V) last = sample_find<T>(x, p, row, false, false, (uint64_t)k, 0.0, hist, share);
    auto total = [&](double least) {
        uint64_t s = 0;
        for (int i = tid; i < p.V; i += SAMPLE_THREADS) {
            const float f = sample_clean((float)x[i]);
            const uint64_t key = sample_key(f, i);
            if (key < last) continue;
            const double m = row.mass(f);
            if (m >= least || key == best) s += row.units(m);
        }
        return sample_block_sum(s, scratch);
    };
    const float top_p = p.top_p ? p.top_p[r] : 1.0f;
    if (top_p < 1.0f) {
        const double limit = (double)top_p * (double)total(0.0);
        const uint64_t at = limit > 0.0 ? sample_find<T>(x, p, row, true, false, 0, limit, hist, share) : best;
        last = at > last ? at : last;
    }
    const float min_p = p.min_p ? p.min_p[r] : 0.0f;
    const uint64_t z = total(min_p > 0.0f ? (double)min_p : 0.0);
    float u = p.uniforms[r];
    u = u > 0.0f ? (u < 1.0f ? u : 1.0f - 5.9604644775390625e-8f) : 0.0f;
    const uint64_t at = sample_find<T>(x, p, row, true, true, 0, (double)u * (double)z, hist, share);
    if (tid == 0) {
        const int i = (int)~(uint32_t)at;
        p.token[r] = i;
        if (p.logprob) p.logprob[r] = (float)(row.exponent(sample_clean((float)x[i])) - log((double)z / row.unit));
    }
}

static inline int sample_shift(int V)
{
    int bits = 0;
    while (((int64_t)1 << bits) <= V) ++bits;            // V < 2^bits
    return 62 - bits < 52 ? 62 - bits : 52;
}

template <class T>
static void sample_launch(const SampleArgs& p, hipStream_t s)
{
    hipLaunchKernelGGL((sample_kernel<T>), dim3((unsigned)p.rows), dim3(SAMPLE_THREADS), 0, s, p);
}

}  // namespace seedinf
