// Sampling with temperature, top-k, top-p and min-p from one given uniform a row.
//
// The choices of a row are ordered by (logit descending, index ascending); every filter keeps a prefix of that order.
// An element's place in it is a 64-bit key, the logit's bits in an order that integers have, then the inverted index:
// larger key = earlier.  Masses are computed in 64 bits and added as 64-bit integers: a sum's value does not depend on
// the order of its terms, so neither does a choice.  Kernels, by the number of choices (sample_launch):
//   lanes  up to 64: a choice a lane, ranks by counting.
//   row    a workgroup a row: one pass over the row adds every choice's mass to a histogram over the logit (2048 bins of
//          1/16 of a temperature); what the filters and the draw ask for is then known up to a few bins; a second pass
//          collects those bins' choices, which are sorted and searched.  A row that top-k or min-p leaves few choices is
//          read once: those go into a list that takes the row's place.
//          Where the bins hold more choices than fit (logits that are all but equal), the questions are answered one
//          by one instead, by radix searches in a bin (sample_find, over the row, with the histogram's masses; 64 x 50001
//          within a hundredth of a temperature: 151 us, with top-p 217, where spread logits take 40).
// What bounds a row: the operations in 64 bits and the LDS additions of the first pass, then some twenty dependent phases
// of 1 - 3 us; few rows leave most compute units idle (64 x 50001 bf16: 44 - 53 us; 4 x 32000 fp32, top-k 50: 24 us).  256 rows of
// 131072 fp32, top-k 1000: 70 us, 1.9 TB/s.  4096 rows of 18: 5.4 us, a launch's own time.
#pragma once
#include <atomic>
#include <cfloat>
#include <type_traits>

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

constexpr int SAMPLE_BITS = 11, SAMPLE_BINS = 1 << SAMPLE_BITS;

// ---- reductions over a workgroup of NT threads; `scratch`: NT / 64 values ----
template <int NT, class V, class F>
__device__ __forceinline__ V sample_reduce(V v, V* scratch, F join)
{
    auto other = [](V x, int off) {
        if constexpr (sizeof(V) == 8) { const uint64_t u = shfl_xor64(__builtin_bit_cast(uint64_t, x), off); return __builtin_bit_cast(V, u); }
        else return __shfl_xor(x, off, 64);
    };
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = join(v, other(v, off));
    __syncthreads();                                         // the previous reduction's readers are done
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    V r = scratch[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) r = join(r, scratch[i]);
    return r;
}

// Inclusive running sums of a[0 .. n) in place, n <= NT * PER, always added in the same order.
template <int NT, int PER, class V>
__device__ __forceinline__ void sample_scan(V* a, int n, V* scratch)
{
    const int tid = threadIdx.x, lane = tid & 63;
    V x[PER], s = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int at = tid * PER + i;
        if (at < n) s += a[at];
        x[i] = s;
    }
    V run = s;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const V o = __shfl_up(run, off, 64);
        if (lane >= off) run += o;
    }
    __syncthreads();
    if (lane == 63) scratch[tid >> 6] = run;
    __syncthreads();
    V before = run - s;
    if constexpr (sizeof(V) == 8) { before = __shfl_up(run, 1, 64); if (lane == 0) before = 0; }      // (double: a difference would round)
    V waves = 0;
    for (int w = 0; w < (tid >> 6); ++w) waves += scratch[w];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int at = tid * PER + i;
        if (at < n) a[at] = waves + before + x[i];
    }
    __syncthreads();
}

// The first place of [from, to) that cond, which holds for all behind one that it holds for, holds for; `none` if there
// is none.  At most 4096 places: the 64 lanes look at the ends of as many parts, then at one part.  Every wavefront
// for itself, without barriers.
template <class F> __device__ __forceinline__ int sample_first_of(int from, int to, int none, F cond)
{
    const int n = to - from, part = (n + 63) / 64, lane = threadIdx.x & 63;
    if (n <= 0) return none;
    uint64_t some = __ballot(cond(from + min(lane * part + part, n) - 1));
    if (!some) return none;
    from += (int)__builtin_ctzll(some) * part;
    some = __ballot(cond(min(from + lane, to - 1)));
    return some ? min(from + (int)__builtin_ctzll(some), to - 1) : from + part - 1;      // (there is one, but for a sum's last bit)
}

// ---- a row of memory: 16-byte vectors between a head and a tail of single elements ----
template <class T> struct SampleMem {
    static constexpr int VEC = 16 / sizeof(T);
    const T* x;
    int V, head, vecs;
    __device__ __forceinline__ SampleMem(const T* x_, int V_) : x(x_), V(V_)
    {
        head = min(V, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T));
        vecs = (V - head) / VEC;
    }
    // f(value, index) for every element of tiles from .. to (NT * U vectors each; the head and the tail are tile 0's), in
    // any order.  A tile is on its way while the one before it is worked on.
    template <int NT, int U, class F> __device__ __forceinline__ void sweep(int from, int to, F f) const
    {
        const u32x4* body = (const u32x4*)(x + head);
        u32x4 v[U], next[U];
        auto load = [&](int tile, u32x4 (&to)[U]) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = (tile * U + u) * NT + (int)threadIdx.x;
                if (i < vecs) to[u] = body[i];
            }
        };
        load(from, v);
        for (int t = from; t < to; ++t) {
            if (t + 1 < to) load(t + 1, next);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = (t * U + u) * NT + (int)threadIdx.x;
                if (at < vecs) {
                    const int i = head + at * VEC;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const uint32_t w = v[u][sizeof(T) == 4 ? e : e / 2];
                        if constexpr (sizeof(T) == 4) f(__builtin_bit_cast(float, w), i + e);
                        else f(e & 1 ? bf16_hi_f32(w) : bf16_lo_f32(w), i + e);
                    }
                }
                v[u] = next[u];
            }
        }
        if (from == 0) {
            if ((int)threadIdx.x < head) f((float)x[threadIdx.x], (int)threadIdx.x);
            const int i = head + vecs * VEC + (int)threadIdx.x;
            if (i < V) f((float)x[i], i);
        }
    }
    // put(index, place) for the elements that wanted(value) holds for, each with a place of its own, from `*n` (in LDS) on,
    // which counts them.  A thread asks for its elements of a tile at once, without a branch.
    template <int NT, int U, class W, class F> __device__ __forceinline__ void gather(int tiles, int* n, W wanted, F put) const
    {
        static_assert(U * VEC <= 32, "");
        const u32x4* body = (const u32x4*)(x + head);
        u32x4 v[U], next[U];
        auto load = [&](int tile, u32x4 (&to)[U]) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = (tile * U + u) * NT + (int)threadIdx.x;
                if (i < vecs) to[u] = body[i];
            }
        };
        load(0, v);
        for (int t = 0; t < tiles; ++t) {
            if (t + 1 < tiles) load(t + 1, next);
            const int first = t * U * NT + (int)threadIdx.x;
            uint32_t mine = 0;                               // a bit an element
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const uint32_t w = v[u][sizeof(T) == 4 ? e : e / 2];
                    const float f = sizeof(T) == 4 ? __builtin_bit_cast(float, w) : (e & 1 ? bf16_hi_f32(w) : bf16_lo_f32(w));
                    mine |= (uint32_t)((first + u * NT < vecs) & wanted(f)) << (u * VEC + e);
                }
            if (mine) {
                int at = atomicAdd(n, __popc(mine));
                for (; mine; mine &= mine - 1, ++at) {
                    const int bit = __builtin_ctz(mine);
                    put(head + (first + bit / VEC * NT) * VEC + bit % VEC, at);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = next[u];
        }
        auto one = [&](int i) { if (wanted((float)x[i])) put(i, atomicAdd(n, 1)); };
        if ((int)threadIdx.x < head) one((int)threadIdx.x);
        const int i = head + vecs * VEC + (int)threadIdx.x;
        if (i < V) one(i);
    }
    template <int NT, int U> __device__ __forceinline__ int tiles() const { return max(1, (vecs + NT * U - 1) / (NT * U)); }
};

// ---- a workgroup a row ----

// The histogram's bins, from the first of the order on: u = 16 (16 - (x - centre) / T), bin floor(u).  Logits up to 16
// temperatures above the centre and 112 below are in it; those further below have less than 2^-160 of the mass, which
// is none; those above make the centre be chosen anew.  A choice's mass is that of its bin's lower edge, exp(16 -
// (bin + 1) / 16) of the centre's, times exp((bin + 1 - u) / 16) in [1, 1.0645), in units of 2^-38: V up to 2^24 of
// them stay below 2^63.  A pass over a row is bound by its operations in 64 bits (a wavefront's takes 8 cycles), so
// they are few: 11 a choice.  place() is u - 1/2; adding 1.5 * 2^52 rounds it to the bin, in the sum's low bits (a place
// on an edge goes to one side or the other, always the same one); what is left, c in [-1/2, 1/2], is the exponential's.
struct SampleBins {
    static constexpr double ROUND = 6755399441055744.0;
    double inv_t, centre, B;     // B = 16 / T
    __device__ __forceinline__ double place(float x) const { return fma(centre - (double)x, B, 255.5); }
    __device__ __forceinline__ static int bin(double v)      // -1: none (NaN's, too)
    {
        const uint64_t b = __builtin_bit_cast(uint64_t, v + ROUND) - __builtin_bit_cast(uint64_t, ROUND);
        return b < (uint64_t)SAMPLE_BINS ? (int)b : -1;
    }
    // exp((c + 1/2) / 16) by the polynomial of degree 5 through the six Chebyshev nodes (off by less than 2^-44), in units
    // of 2^-38: the last sum's rounding, 2^14 being in its constant
    __device__ __forceinline__ static uint64_t units(double v)
    {
        const double c = ((v + ROUND) - ROUND) - v;
        double e = 8.199845889429414e-09;
        e = fma(e, c, 6.559968227281715e-07);
        e = fma(e, c, 4.198174669759914e-05);
        e = fma(e, c, 0.0020151238397688406);
        e = fma(e, c, 0.06448396296869428);
        e = fma(e, c, 16384.0 + 1.0317434074991443);
        return __builtin_bit_cast(uint64_t, e) - __builtin_bit_cast(uint64_t, 16384.0);
    }
    __device__ __forceinline__ static double edge(int bin) { return exp(16.0 - (bin + 1) * 0.0625) * (1.0 / 274877906944.0); }
    __device__ __forceinline__ static double mass(double v) { return (double)units(v) * edge(bin(v)); }
};

// ---- radix searches: where a bin holds more choices than the list, several passes a question ----

// One place of the order inside bin `bin`: the first choice at which the running count (mass = false) reaches `count`, or
// the bin's running mass, in the bin's units, makes reached(units) true; the bin's last choice if there is none.  Returns its
// key; `upto`: the count or the units up to and with it, 0 if the bin has no choice.  value(f): what a logit counts as.
// Digits of the key from the top, up to 11 bits a pass over the row: three for the logit, those that V needs for the index.
// A thread adds its choices up while they have the same digit (in rows of equal logits all have).
template <class T, int NT, class V, class F>
__device__ __forceinline__ uint64_t sample_find(const SampleMem<T>& x, const SampleBins& bins, int bin, bool mass, uint64_t count, V value, F reached,
                                                uint64_t* hist, uint64_t* scratch, uint64_t& upto)
{
    const int tid = threadIdx.x, index_bits = 32 - __builtin_clz(max(x.V - 1, 1));
    uint64_t prefix = 0, before = 0;
    int low = 64;                                            // key bits below `low` are not yet known
    while (low > 0) {
        if (low == 32 && index_bits < 32) {                  // (the index is inverted: ones above its bits)
            prefix = prefix << (32 - index_bits) | ((1ull << (32 - index_bits)) - 1);
            low = index_bits;
        }
        const int w = low > 32 ? min(SAMPLE_BITS, low - 32) : min(SAMPLE_BITS, low), at = low - w, digits = 1 << w;
        __syncthreads();                                     // (the previous pass's readers are done)
        for (int i = tid; i < SAMPLE_BINS; i += NT) hist[i] = 0;
        __syncthreads();
        int digit = 0;
        uint64_t sum = 0;
        x.template sweep<NT, 2>(0, x.template tiles<NT, 2>(), [&](float f, int i) {
            f = value(f);
            const uint64_t key = sample_key(f + 0.0f, i);
            if (low < 64 && (key >> low) != prefix) return;
            const double v = mass || low > 32 ? bins.place(f) : 0.0;
            if (low > 32 && bins.bin(v) != bin) return;      // (with the logit's digits known, all are in the bin)
            const int d = digits - 1 - (int)((key >> at) & (digits - 1));    // (larger keys first)
            if (d != digit) {
                if (sum) atomicAdd((unsigned long long*)&hist[digit], (unsigned long long)sum);
                digit = d; sum = 0;
            }
            sum += mass ? bins.units(v) : 1;
        });
        if (sum) atomicAdd((unsigned long long*)&hist[digit], (unsigned long long)sum);
        __syncthreads();
        sample_scan<NT, SAMPLE_BINS / NT>(hist, SAMPLE_BINS, scratch);
        const uint64_t all = hist[digits - 1];
        if (all == 0) { upto = 0; __syncthreads(); return 0; }
        const int d = sample_first_of(0, digits, digits - 1, [&](int b) {
            const uint64_t run = before + hist[b];
            return hist[b] == all || (mass ? reached(run) : run >= count);
        });
        upto = before + hist[d];
        if (d > 0) before += hist[d - 1];
        prefix = prefix << w | (uint64_t)(digits - 1 - d);
        low = at;
    }
    __syncthreads();
    return prefix;
}

template <int CAP> struct SampleLds {
    uint64_t hist[SAMPLE_BINS + 64];                         // masses; then, as doubles, their running sums (64 places for what is in no bin)
    uint32_t count[SAMPLE_BINS];                             // choices; then their running sums
    uint64_t list[CAP];                                      // keys of the collected choices
    double run[CAP];                                         // running sums over them
    uint32_t wanted[SAMPLE_BINS / 32], near[SAMPLE_BINS / 32];       // bits of the bins to collect; of those and their neighbours
    uint64_t scratch[16];
    int found, n;
};

template <class T, int NT, int CAP>
__global__ __launch_bounds__(NT) void sample_row_kernel(SampleArgs p)
{
    constexpr int U = 4, NB = SAMPLE_BINS;
    extern __shared__ __attribute__((aligned(16))) char sample_lds[];
    SampleLds<CAP>& l = *(SampleLds<CAP>*)sample_lds;
    double* const cum = (double*)l.hist;
    const int r = blockIdx.x, tid = threadIdx.x;
    const SampleMem<T> row((const T*)p.logits + (int64_t)r * p.stride, p.V);
    const float temp = p.temperature ? p.temperature[r] : 1.0f;
    const int tiles = row.template tiles<NT, U>();
    auto larger = [](uint64_t a, uint64_t b) { return a > b ? a : b; };
    auto first_key = [&]() {                                 // the first of the order
        uint64_t best = 0;
        row.template sweep<NT, U>(0, tiles, [&](float f, int i) { best = larger(best, sample_key(sample_clean(f), i)); });
        return sample_reduce<NT>(best, l.scratch, larger);
    };
    auto largest = [&](float f) { return sample_reduce<NT>(f, (float*)l.scratch, [](float a, float b) { return fmaxf(a, b); }); };
    auto value = [](uint64_t key) {                          // the logit of a key
        const uint32_t b = (uint32_t)(key >> 32);
        return __builtin_bit_cast(float, (b >> 31) ? b & 0x7fffffffu : ~b);
    };
    const int k0 = p.top_k ? p.top_k[r] : 0;
    float min_p = p.min_p ? p.min_p[r] : 0.0f;
    if (!(min_p > 0.0f)) min_p = 0.0f;
    const bool greedy = !(temp > 0.0f) || k0 == 1 || min_p > 1.0f;       // one choice is kept
    if (greedy) {
        const uint64_t best = first_key();
        const bool none = value(best) == -INFINITY;
        if (tid == 0) { p.token[r] = none ? -1 : (int)~(uint32_t)best; if (p.logprob) p.logprob[r] = none ? -INFINITY : 0.0f; }
        return;
    }
    float top_p = p.top_p ? p.top_p[r] : 1.0f;
    if (!(top_p < 1.0f)) top_p = 1.0f;
    float u01 = p.uniforms[r];
    u01 = u01 > 0.0f ? (u01 < 1.0f ? u01 : 1.0f - 5.9604644775390625e-8f) : 0.0f;
    const int k = k0 > 0 && k0 < p.V ? k0 : 0;               // 0: off
    const bool all_mass = top_p < 1.0f && k == 0;            // the mass of every choice is asked for

    SampleBins bins;
    bins.inv_t = 1.0 / (double)temp;
    bins.B = 16.0 * bins.inv_t;
    // Choices below `cut` (a logit, a little too low rather than too high) no longer matter.
    float cut;
    float top = -INFINITY;                                   // the largest logit, as far as it is known (NaN is none: fmaxf)
    row.template sweep<NT, U>(0, 1, [&](float f, int) { top = fmaxf(top, f); });
    top = largest(top);
    bool inf_row = top == INFINITY;                          // +inf among the logits: those are the choices, all equal
    // (below the place's own logit by more than its roundings)
    auto logit_at = [&](double u) {
        const double x = bins.centre + (256.0 - u) * 0.0625 * (double)temp;
        return (float)(x - fabs(x) * 1e-6 - fabs(bins.centre) * 1e-6 - 1e-30);
    };
    // The end of the bins up to which the first k choices counted in l.count lie, NB if there are not as many.
    auto k_end = [&]() {
        __syncthreads();
        uint32_t mine = 0;
        for (int i = tid * (NB / NT); i < (tid + 1) * (NB / NT); ++i) mine += l.count[i];
        uint32_t run = mine;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) { const uint32_t o = __shfl_up(run, off, 64); if ((tid & 63) >= off) run += o; }
        uint32_t* waves = (uint32_t*)l.scratch;
        if (tid == 0) l.found = NB;
        if ((tid & 63) == 63) waves[tid >> 6] = run;
        __syncthreads();
        for (int w = 0; w < (tid >> 6); ++w) run += waves[w];
        if (run >= (uint32_t)k && run - mine < (uint32_t)k) l.found = (tid + 1) * (NB / NT);
        __syncthreads();
        return l.found;
    };
    auto clear = [&]() {
        __syncthreads();
        for (int i = tid; i < NB; i += NT) { l.hist[i] = 0; l.count[i] = 0; }
        __syncthreads();
    };
    auto add = [&](float f) {                                // a choice to the histogram
        const double v = bins.place(f);
        const int bin = bins.bin(v);
        if (bin >= 0) {
            atomicAdd((unsigned long long*)&l.hist[bin], (unsigned long long)bins.units(v));
            if (k) atomicAdd(&l.count[bin], 1u);
        }
    };
    // Where a filter leaves few choices whatever the rest of the row, the row is read once and those that may be among
    // them are kept in a list: all that are not behind the k-th, or not below min-p, of what was read so far.  The mass of
    // the others is not asked for.  If the list does not hold them, the row is taken as a whole below.
    uint64_t* const cand = (uint64_t*)l.run;
    int cands = 0;
    bool listed = tiles > 1 && !inf_row && top != -INFINITY && (k ? k <= CAP / 4 : min_p > 0.0f && !all_mass);
    if (listed) {
        bins.centre = (double)top;
        cut = -FLT_MAX;
        auto narrow = [&]() {                                // the cut, from the counts (k) or the largest logit (min-p)
            if (k) { const int e = k_end(); if (e < NB) cut = fmaxf(cut, logit_at((double)e)); }
            if (min_p > 0.0f && (k == 0 || !(top_p < 1.0f))) cut = fmaxf(cut, logit_at(257.0 - 16.0 * log((double)min_p)));
        };
        if (k) {
            clear();
            row.template sweep<NT, U>(0, 1, [&](float f, int) { const int bin = bins.bin(bins.place(f)); if (bin >= 0) atomicAdd(&l.count[bin], 1u); });
        }
        narrow();
        __syncthreads();
        if (tid == 0) l.n = 0;
        __syncthreads();
        // Behind t tiles another t add about k: there the cut is looked at again, the list then holds some 2 k.
        for (int t = 0, end; t < tiles; t = end) {
            end = min(tiles, max(t + 1, t * 2));
            row.template sweep<NT, U>(t, end, [&](float f, int i) {
                if (f >= cut) {
                    const int at = atomicAdd(&l.n, 1);
                    if (at < CAP) cand[at] = sample_key(f + 0.0f, i);
                }
            });
            __syncthreads();
            cands = l.n;
            __syncthreads();                                 // (read by all before the next tiles add to it)
            if (cands > CAP) break;
            if (cands <= 3 * CAP / 8) {
                if (end < tiles) continue;
                top = -INFINITY;                             // few enough at the end: the centre at the largest is all that is wanted
                for (int i = tid; i < cands; i += NT) top = fmaxf(top, value(cand[i]));
                top = largest(top);
                bins.centre = (double)top;
            } else {                                         // the centre at the largest so far, the cut anew, and out with what is below it
                uint64_t mine[CAP / NT];
                top = -INFINITY;
#pragma unroll
                for (int j = 0; j < CAP / NT; ++j) {
                    mine[j] = tid + j * NT < cands ? cand[tid + j * NT] : 0;
                    if (mine[j]) top = fmaxf(top, value(mine[j]));
                }
                top = largest(top);
                if (top == INFINITY) break;
                bins.centre = (double)top;
                clear();
                if (k)
#pragma unroll
                    for (int j = 0; j < CAP / NT; ++j)
                        if (mine[j]) { const int bin = bins.bin(bins.place(value(mine[j]))); if (bin >= 0) atomicAdd(&l.count[bin], 1u); }
                narrow();
                __syncthreads();
                if (tid == 0) l.n = 0;
                __syncthreads();
#pragma unroll
                for (int j = 0; j < CAP / NT; ++j) if (mine[j] && value(mine[j]) >= cut) cand[atomicAdd(&l.n, 1)] = mine[j];
                __syncthreads();
                cands = l.n;
                __syncthreads();
            }
        }
        listed = cands <= CAP && top != INFINITY;
        if (listed) {
            clear();
            for (int i = tid; i < cands; i += NT) add(value(cand[i]));
        }
        __syncthreads();
    }
    for (int attempt = 0; !listed; ++attempt) {
        // the centre: the largest logit of the first tile; if one is found far above it, the largest of all
        inf_row = top == INFINITY;
        if (top == -INFINITY && attempt > 0) {               // no choice at all
            if (tid == 0) { p.token[r] = -1; if (p.logprob) p.logprob[r] = -INFINITY; }
            return;
        }
        bins.centre = inf_row || top == -INFINITY ? 0.0 : (double)top;
        // min-p without top-p: nothing below it is asked for (the largest logit is not below the centre)
        cut = min_p > 0.0f && !all_mass && !(k && top_p < 1.0f) ? logit_at(257.0 - 16.0 * log((double)min_p)) : -INFINITY;
        clear();
        float seen = -INFINITY;
        for (int t = 0; t < tiles; t = t ? tiles : 1) {
            // (nothing is left out: without a branch the choices' operations overlap; each lane has a place of its own for what is in no bin)
            if (cut == -INFINITY && !inf_row && !k) {
                row.template sweep<NT, U>(0, tiles, [&](float f, int) {
                    seen = fmaxf(seen, f);
                    const double v = bins.place(f);
                    const int bin = bins.bin(v);
                    atomicAdd((unsigned long long*)&l.hist[bin >= 0 ? bin : NB + (tid & 63)], (unsigned long long)bins.units(v));
                });
                break;
            }
            row.template sweep<NT, U>(t, t ? tiles : 1, [&](float f, int i) {
                seen = fmaxf(seen, f);
                if (!(f >= cut)) return;                     // (NaN neither)
                if (inf_row) f = f == INFINITY ? 0.0f : -INFINITY;
                add(f);
            });
            // what is behind the k-th choice of one tile is behind the k-th of all
            if (k && t == 0 && tiles > 2) {
                const int e = k_end();
                if (e < NB) cut = fmaxf(cut, logit_at((double)e));
                __syncthreads();
            }
        }
        const float was = top;
        top = largest(seen);
        // nothing lies above the bins (and the centre was a logit, the row of the kind that was assumed)
        if (attempt > 0 ? top != -INFINITY : was != -INFINITY && (top == INFINITY) == inf_row && (inf_row || bins.bin(bins.place(top)) >= 0)) break;
    }
    // running sums over the bins
    for (int i = tid; i < NB; i += NT) { const uint64_t h = l.hist[i]; cum[i] = h ? (double)h * SampleBins::edge(i) : 0.0; }
    __syncthreads();
    sample_scan<NT, NB / NT>(cum, NB, (double*)l.scratch);
    if (k) sample_scan<NT, NB / NT>(l.count, NB, (uint32_t*)l.scratch);
    auto first_bin = [&](auto cond) { return sample_first_of(0, NB, NB - 1, cond); };
    auto before = [&](int b) { return b > 0 ? cum[b - 1] : 0.0; };
    const double z_all = cum[NB - 1];
    // The last kept choice lies in bin kb (top-k), between pb0 and pb1 (top-p), in mb (min-p); what is drawn between db0 and db1.
    const bool k_on = k && l.count[NB - 1] >= (uint32_t)k;   // (choices that are in no bin have no mass)
    const int kb = k_on ? first_bin([&](int b) { return l.count[b] >= (uint32_t)k; }) : NB - 1;
    const bool k_part = k_on && l.count[kb] > (uint32_t)k;   // the bin is cut
    const double zk0 = k_on ? before(kb) : z_all, zk1 = k_on ? cum[kb] : z_all;
    int pb0 = NB - 1, pb1 = NB - 1;
    if (top_p < 1.0f) {
        const double t0 = (double)top_p * (k_part ? zk0 : zk1), t1 = (double)top_p * zk1;
        pb0 = first_bin([&](int b) { return cum[b] >= t0 && cum[b] > 0.0; });
        pb1 = first_bin([&](int b) { return cum[b] >= t1 && cum[b] > 0.0; });
    }
    const double m_place = min_p > 0.0f ? bins.place(inf_row ? 0.0f : top) - 16.0 * log((double)min_p) : INFINITY;    // kept: place <= m_place
    const int mb = m_place < (double)NB - 0.5 ? max(bins.bin(m_place), 0) : NB - 1;
    const int e0 = min(kb, min(pb0, mb)), e1 = min(kb, min(pb1, mb));
    const double d0 = (double)u01 * before(e0), d1 = (double)u01 * cum[e1];
    const int db0 = first_bin([&](int b) { return cum[b] > d0; }), db1 = first_bin([&](int b) { return cum[b] > d1; });
    // collect the choices of those bins (and the first bin's, so that there is always one)
    for (int i = tid; i < NB / 32; i += NT) l.wanted[i] = l.near[i] = 0;
    if (tid == 0) l.n = 0;
    __syncthreads();
    const int fb = max(bins.bin(bins.place(inf_row ? 0.0f : top)), 0);
    auto want = [&](int from, int to) {
        for (int b = max(from - 1, 0) + tid; b <= min(to + 1, NB - 1); b += NT) {
            atomicOr(&l.near[b >> 5], 1u << (b & 31));
            if (b >= from && b <= to) atomicOr(&l.wanted[b >> 5], 1u << (b & 31));
        }
    };
    if (k_part) want(kb, kb);
    if (top_p < 1.0f) want(pb0, pb1);
    if (mb < NB - 1) want(mb, mb);
    want(db0, db1);
    want(fb, fb);
    __syncthreads();
    // In 32 bits a place is within 2^-10 of a bin of what it is in 64 (the centre is a logit), but for temperatures whose
    // inverse leaves 32 bits, or so large that logits whose difference does may share the bins.
    const float near_centre = (float)bins.centre, near_b = (float)bins.B;
    const bool far = !(temp > 1e-30f && temp < 1e36f);
    auto near = [&](float f) {
        const int b = (int)fminf(fmaxf(fmaf(near_centre - f, near_b, 256.0f), 0.0f), (float)(NB - 1));
        return (l.near[b >> 5] >> (b & 31) & 1) | far;
    };
    auto wanted = [&](float f) {
        const int bin = bins.bin(bins.place(f));
        return (bin >= 0) & (l.wanted[max(bin, 0) >> 5] >> (bin & 31) & 1);
    };
    auto collect = [&](float f, int i) {
        const int at = atomicAdd(&l.n, 1);
        if (at < CAP) l.list[at] = sample_key(f + 0.0f, i);
    };
    if (listed) {
        for (int i = tid; i < cands; i += NT)
            if (const float f = value(cand[i]); wanted(f)) collect(f, (int)~(uint32_t)cand[i]);
    } else if (inf_row) {
        row.template sweep<NT, U>(0, tiles, [&](float f, int i) { if (f == INFINITY) collect(0.0f, i); });
    } else {
        // the indices of those that are near, then of these the wanted ones (900 of 50001: 12.5 us; directly, 16 us)
        int* const some = (int*)l.run;
        row.template gather<NT, U>(tiles, &l.n, near, [&](int i, int at) { if (at < 2 * CAP) some[at] = i; });
        __syncthreads();
        const int m = l.n;
        __syncthreads();
        if (tid == 0) l.n = 0;
        __syncthreads();
        if (m <= 2 * CAP) {
            for (int i = tid; i < m; i += NT)
                if (const float f = (float)row.x[some[i]]; wanted(f)) collect(f, some[i]);
        } else row.template sweep<NT, U>(0, tiles, [&](float f, int i) { if (wanted(f)) collect(f, i); });
    }
    __syncthreads();
    const int n = l.n;
    if (n > CAP) {                                           // (uniform): the questions below, answered by searches in the bins
        uint64_t* const hist = l.list;                       // (the list and its running sums: 2048 places at least)
        static_assert(2 * CAP >= SAMPLE_BINS, "");
        auto as = [&](float f) { f = sample_clean(f); return inf_row ? (f == INFINITY ? 0.0f : -INFINITY) : f; };
        auto units_of = [&](int b, auto counts) {            // of the choices of bin b that counts(key, place) holds for
            uint64_t sum = 0;
            row.template sweep<NT, 2>(0, row.template tiles<NT, 2>(), [&](float f, int i) {
                f = as(f);
                const double v = bins.place(f);
                if (bins.bin(v) == b && counts(sample_key(f + 0.0f, i), v)) sum += bins.units(v);
            });
            return (double)sample_reduce<NT>(sum, l.scratch, [](uint64_t a, uint64_t b) { return a + b; });
        };
        double z = z_all;
        int end = NB;
        uint64_t upto = 0;
        __syncthreads();
        if (k_on) {
            z = zk1; end = kb;
            if (k_part) {
                const uint64_t last = sample_find<T, NT>(row, bins, kb, false, (uint64_t)((uint32_t)k - (kb > 0 ? l.count[kb - 1] : 0u)), as,
                                                         [](uint64_t) { return false; }, hist, l.scratch, upto);
                z = before(kb) + units_of(kb, [&](uint64_t key, double) { return key >= last; }) * SampleBins::edge(kb);
            }
        }
        if (top_p < 1.0f) {
            const double limit = (double)top_p * z;
            const int b = first_bin([&](int b) { return cum[b] >= limit && cum[b] > 0.0; });
            const double from = before(b), edge = SampleBins::edge(b);
            sample_find<T, NT>(row, bins, b, true, 0, as, [&](uint64_t run) { return from + (double)run * edge >= limit; }, hist, l.scratch, upto);
            const double zp = from + (double)upto * edge;
            if (b < end || (b == end && zp < z)) { end = b; z = zp; }
        }
        if (mb < NB - 1 && mb <= end) {
            const double zm = before(mb) + units_of(mb, [&](uint64_t, double v) { return v <= m_place; }) * SampleBins::edge(mb);
            if (mb < end || zm < z) { end = mb; z = zm; }
        }
        const double one = bins.mass(bins.place(inf_row ? 0.0f : top));
        if (!(z >= one)) z = one;
        const double limit = (double)u01 * z;
        uint64_t key;
        int b = first_bin([&](int b) { return cum[b] > limit; });
        do {                                                 // (a running sum's last bit may point behind the last choice)
            const double from = before(b), edge = SampleBins::edge(b);
            key = sample_find<T, NT>(row, bins, b, true, 0, as, [&](uint64_t run) { return from + (double)run * edge > limit; }, hist, l.scratch, upto);
        } while (upto == 0 && b-- > 0);
        if (tid == 0) {
            p.token[r] = min((int)(~(uint32_t)key & 0x7fffffffu), p.V - 1);
            if (p.logprob) p.logprob[r] = (float)log(bins.mass(bins.place(value(key))) / z);
        }
        return;
    }
    // sort them, larger keys first: up to 256 by counting those in front of each, with several threads for one where there are
    // as many (266: 5.2 us; 700: 33 us), more by a bitonic network (places behind n: key 0, behind all), up to NT of them a
    // key a thread, with exchanges between lanes, and through memory only between wavefronts (266: 6.5 us; 700: 8 us)
    if (n <= 256) {
        const int some = max(64, (n + 63) & ~63), parts = NT / some, per = (n + parts - 1) / parts, part = tid / some, me = tid - part * some;
        int* const rank = (int*)l.run;
        if (tid < n) rank[tid] = 0;
        __syncthreads();
        const uint64_t mine = me < n ? l.list[me] : 0;
        int in_front = 0;
        for (int i = part * per; i < min(n, (part + 1) * per); ++i) in_front += l.list[i] > mine;
        if (part < parts && me < n) atomicAdd(&rank[me], in_front);
        __syncthreads();
        if (tid < n) l.list[rank[tid]] = mine;
    } else if (n <= NT) {
        int size = 64;
        while (size < n) size *= 2;
        uint64_t mine = tid < n ? l.list[tid] : 0;
        uint64_t* buffer[2] = {(uint64_t*)l.run, l.list};
        int turn = 0;
        for (int a = 2; a <= size; a *= 2)
            for (int b = a / 2; b > 0; b /= 2) {
                uint64_t other;
                if (b >= 64) {
                    uint64_t* const to = turn ? buffer[1] : buffer[0];       // (in turn: one barrier an exchange)
                    turn ^= 1;
                    to[tid] = mine;
                    __syncthreads();
                    other = to[tid ^ b];
                } else other = shfl_xor64(mine, b);
                if ((mine < other) == (((tid & b) == 0) == ((tid & a) == 0))) mine = other;
            }
        __syncthreads();
        if (tid < n) l.list[tid] = mine;
    } else {
        int size = 2 * NT;
        while (size < n) size *= 2;
        for (int i = n + tid; i < size; i += NT) l.list[i] = 0;
        for (int a = 2; a <= size; a *= 2)
            for (int b = a / 2; b > 0; b /= 2) {
                __syncthreads();
                for (int i = tid; i < size / 2; i += NT) {
                    const int x = 2 * i - (i & (b - 1)), y = x + b;
                    const uint64_t kx = l.list[x], ky = l.list[y];
                    if ((kx < ky) == ((x & a) == 0)) { l.list[x] = ky; l.list[y] = kx; }
                }
            }
    }
    __syncthreads();
    // each one's mass; then the running sums over the list, and from them those over the whole order
    auto place_of = [&](uint64_t key) { return bins.place(value(key)); };
    for (int i = tid; i < n; i += NT) l.run[i] = bins.mass(place_of(l.list[i]));
    __syncthreads();
    sample_scan<NT, CAP / NT>(l.run, n, (double*)l.scratch);
    if (tid >= 64) return;                                   // the rest is one wavefront's
    auto bin_of = [&](int i) { return bins.bin(place_of(l.list[i])); };
    auto range = [&](int b, int& from, int& to) {            // [from, to): the list's part of bin b
        from = sample_first_of(0, n, n, [&](int i) { return bin_of(i) >= b; });
        to = sample_first_of(from, n, n, [&](int i) { return bin_of(i) > b; });
    };
    auto sum_at = [&](int i, int from, int b) { return before(b) + (l.run[i] - (from > 0 ? l.run[from - 1] : 0.0)); };
    double z = z_all;                                        // mass of the kept ones
    int end = NB;                                            // bin that the last kept one lies in
    int f, t;
    if (k_on) {
        z = zk1; end = kb;
        if (k_part) {
            range(kb, f, t);
            const int at = f + (int)((uint32_t)k - (kb > 0 ? l.count[kb - 1] : 0u)) - 1;
            z = sum_at(at, f, kb);
        }
    }
    if (top_p < 1.0f) {
        const double limit = (double)top_p * z;
        const int b = first_bin([&](int b) { return cum[b] >= limit && cum[b] > 0.0; });
        range(b, f, t);
        const int at = sample_first_of(f, t, t - 1, [&](int i) { return sum_at(i, f, b) >= limit; });
        const double zp = f < t ? sum_at(at, f, b) : cum[b];
        if (b < end || (b == end && zp < z)) { end = b; z = zp; }
    }
    if (mb < NB - 1 && mb <= end) {
        range(mb, f, t);
        const int at = sample_first_of(f, t, t, [&](int i) { return place_of(l.list[i]) > m_place; }) - 1;      // the last that is kept
        const double zm = at >= f ? sum_at(at, f, mb) : before(mb);
        if (mb < end || zm < z) { end = mb; z = zm; }
    }
    {                                                        // never fewer than one choice
        const double one = l.run[0];                         // the list begins with the first of the order
        if (!(z >= one)) z = one;
    }
    const double limit = (double)u01 * z;
    const int b = first_bin([&](int b) { return cum[b] > limit; });
    range(b, f, t);
    const int at = sample_first_of(f, t, max(t - 1, 0), [&](int i) { return sum_at(i, f, b) > limit; });
    if (tid == 0) {
        const uint64_t key = l.list[at];
        p.token[r] = (int)~(uint32_t)key;
        if (p.logprob) p.logprob[r] = (float)log(bins.mass(place_of(key)) / z);
    }
}

// ---- up to 64 choices: a choice a lane, L lanes a row ----

// What rows of up to 64 choices compute with.
struct SampleRow {
    float top;                   // the largest logit
    double inv_t;
    double unit;                 // 2^57
    // the equal of an infinite largest logit has mass 1, what is below it and a masked choice none at any temperature
    __device__ __forceinline__ double exponent(float x) const { return x == top ? 0.0 : (x == -INFINITY || top == INFINITY ? -INFINITY : ((double)x - (double)top) * inv_t); }
    __device__ __forceinline__ double mass(float x) const { return exp(exponent(x)); }
    __device__ __forceinline__ uint64_t units(double m) const { return (uint64_t)(m * unit + 0.5); }
};

template <class T, int L>
__global__ __launch_bounds__(256) void sample_lanes_kernel(SampleArgs p)
{
    const int lane = threadIdx.x & 63, me = lane & (L - 1), base = lane & ~(L - 1);
    const int r = blockIdx.x * (256 / L) + threadIdx.x / L;
    const bool here = r < p.rows;                            // (every lane stays for the exchanges)
    const float x = here && me < p.V ? sample_clean((float)((const T*)p.logits)[(int64_t)r * p.stride + me]) : -INFINITY;
    const float temp = here ? (p.temperature ? p.temperature[r] : 1.0f) : 0.0f;
    const int k0 = here && p.top_k ? p.top_k[r] : 0;
    const float top_p = here && p.top_p ? p.top_p[r] : 1.0f, min_p = here && p.min_p ? p.min_p[r] : 0.0f;
    float u = here ? p.uniforms[r] : 0.0f;
    u = u > 0.0f ? (u < 1.0f ? u : 1.0f - 5.9604644775390625e-8f) : 0.0f;
    // my place in the order
    int rank = 0;
    float top = -INFINITY;
    for (int i = 0; i < p.V; ++i) {
        const float o = __shfl(x, base + i, 64);
        rank += o > x || (o == x && i < me);
        top = fmaxf(top, o);
    }
    if (me >= p.V) rank = me;                                // (lanes without a choice: behind all)
    const bool greedy = !(temp > 0.0f);
    SampleRow row;
    row.top = top; row.inv_t = greedy ? 1.0 : 1.0 / (double)temp; row.unit = 144115188075855872.0;      // 2^57
    const double mine = x == -INFINITY ? 0.0 : row.mass(x);
    // in the order: lane j of the row's has the j-th choice
    auto push32 = [&](uint32_t v) { return (uint32_t)__builtin_amdgcn_ds_permute((base + rank) * 4, (int)v); };
    auto push64 = [&](uint64_t v) { return (uint64_t)push32((uint32_t)(v >> 32)) << 32 | push32((uint32_t)v); };
    const int index = (int)push32((uint32_t)me);
    const double m = __builtin_bit_cast(double, push64(__builtin_bit_cast(uint64_t, mine)));
    const double ex = __builtin_bit_cast(double, push64(__builtin_bit_cast(uint64_t, row.exponent(x))));
    uint64_t run = row.units(m);                             // running mass
#pragma unroll
    for (int off = 1; off < L; off <<= 1) {
        const uint32_t lo = __shfl_up((int)(uint32_t)run, off, L), hi = __shfl_up((int)(uint32_t)(run >> 32), off, L);
        if (me >= off) run += (uint64_t)hi << 32 | lo;
    }
    auto at = [&](uint64_t v, int i) { return (uint64_t)(uint32_t)__shfl((int)(uint32_t)(v >> 32), base + i, 64) << 32 | (uint32_t)__shfl((int)(uint32_t)v, base + i, 64); };
    auto first = [&](bool c, int none) {                     // first lane of the row's with c
        const uint64_t b = (__ballot(c) >> base) & (L == 64 ? ~0ull : (1ull << L) - 1);
        return b ? (int)__builtin_ctzll(b) : none;
    };
    int n = greedy ? 1 : (k0 > 0 && k0 < p.V ? k0 : p.V);
    if (top_p < 1.0f) n = min(n, 1 + first((double)run >= (double)top_p * (double)at(run, n - 1), n - 1));
    if (min_p > 0.0f) n = min(n, max(1, first(!(m >= (double)min_p), L)));
    const uint64_t z = at(run, n - 1);
    const int drawn = first((double)run > (double)u * (double)z, n - 1);
    const int token = __shfl(index, base + drawn, 64);
    const double e = __builtin_bit_cast(double, at(__builtin_bit_cast(uint64_t, ex), drawn));
    if (here && me == 0) {
        const bool none = top == -INFINITY;
        p.token[r] = none ? -1 : token;
        if (p.logprob) p.logprob[r] = none ? -INFINITY : greedy ? 0.0f : (float)(e - log((double)z / row.unit));
    }
}

constexpr int SAMPLE_SMALL = 8192;       // choices up to which a row is 256 threads' work

template <class T>
static hipError_t sample_launch(const SampleArgs& p, hipStream_t s)
{
    if (p.V <= 64) {
        auto go = [&](auto lanes) {
            constexpr int L = decltype(lanes)::value;
            hipLaunchKernelGGL((sample_lanes_kernel<T, L>), dim3((unsigned)((p.rows + 256 / L - 1) / (256 / L))), dim3(256), 0, s, p);
        };
        if (p.V <= 8) go(std::integral_constant<int, 8>{});
        else if (p.V <= 16) go(std::integral_constant<int, 16>{});
        else if (p.V <= 32) go(std::integral_constant<int, 32>{});
        else go(std::integral_constant<int, 64>{});
        return hipSuccess;
    }
    if (p.V <= SAMPLE_SMALL) {
        hipLaunchKernelGGL((sample_row_kernel<T, 256, 1024>), dim3((unsigned)p.rows), dim3(256), sizeof(SampleLds<1024>), s, p);
        return hipSuccess;
    }
    constexpr size_t lds = sizeof(SampleLds<4096>);
    static std::atomic<uint64_t> asked{0};
    const hipError_t e = op_allow_lds((const void*)sample_row_kernel<T, 1024, 4096>, lds, asked);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((sample_row_kernel<T, 1024, 4096>), dim3((unsigned)p.rows), dim3(1024), lds, s, p);
    return hipSuccess;
}

}  // namespace seedinf
