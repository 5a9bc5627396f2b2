// Group normalisation with an activation, channels last:
//   y = act((x - mean) / sqrt(var + eps) * weight + bias),
// mean and variance over all points of a row and the channels of a group.
//
// Bound by memory: x in, y out, a few operations a value.  Where a row's values stay in registers between the statistics
// and the result they travel once; mean and variance are always two passes over values that are held (differences to
// the mean, squared), never a difference of sums.  Kernels, by shape (norm_plan):
//   segment   points == 1: a group is a run of channels; a few lanes own it, sums are shuffles.
//   resident  a row (or a slice of its groups) fits a workgroup's registers: read once, written once.
//   split     larger rows: statistics of runs of points, then a second kernel that joins them and reads x again.
//   plain     what is left: slices of more vectors than the split kernel has threads (a group, or the least run of whole
//             groups and vectors, of more than 512 of them), one point a row of groups that no workgroup's registers hold.
#pragma once
#include <algorithm>
#include <numeric>

#include "op_common.h"

namespace seedinf {

struct NormArgs {
    const void* x; void* y;
    const float* weight; const float* bias;      // [channels] or nullptr
    int N, P, C, G;
    float eps;
    int act;
    int vec_params;                              // weight and bias are 16-byte aligned
};

// VEC elements as they are in memory; pairs of bf16 stay one register (as an array of bf16 each element would take one)
template <class T, int VEC> struct alignas(VEC * sizeof(T)) Pack {
    T v[VEC];
    __device__ __forceinline__ float get(int e) const { return (float)v[e]; }
    __device__ __forceinline__ void set(int e, const float* f) { v[e] = (T)f[0]; }
    static constexpr int SET = 1;                // elements a set() takes
};
template <int VEC> struct alignas(VEC * 2) Pack2 {
    uint32_t w[VEC / 2];
    __device__ __forceinline__ float get(int e) const { return e & 1 ? bf16_hi_f32(w[e / 2]) : bf16_lo_f32(w[e / 2]); }
    __device__ __forceinline__ void set(int e, const float* f) { w[e / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2){f[0], f[1]}, bf16x2)); }
    static constexpr int SET = 2;
};
template <> struct Pack<__bf16, 2> : Pack2<2> {};
template <> struct Pack<__bf16, 4> : Pack2<4> {};
template <> struct Pack<__bf16, 8> : Pack2<8> {};

// What is held between two passes is held as it was read: without this the compiler keeps the converted values, twice
// the registers, and half as many workgroups share a compute unit.
template <class T, int VEC>
__device__ __forceinline__ void norm_keep_packed(Pack<T, VEC>& d)
{
    if constexpr (Pack<T, VEC>::SET == 2) {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) asm volatile("" : "+v"(d.w[i]));
    }
}

// d: difference to the mean, a: weight over the deviation; T: what the result is rounded to
template <class T>
__device__ __forceinline__ float norm_finish(float d, float a, float b, int act)
{
    const float v = fmaf(d, a, b);
    if (act == SEED_ACT_RELU) return op_activate<SEED_ACT_RELU, T>(v);
    if (act == SEED_ACT_SILU) return op_activate<SEED_ACT_SILU, T>(v);
    return v;
}

// VEC parameters from channel c (a multiple of VEC) on, `other` where there are none
template <int VEC>
__device__ __forceinline__ void norm_params(const float* w, int c, int aligned, float other, float (&f)[VEC])
{
    if (!w) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = other;
    } else if (VEC % 4 == 0 && aligned) {
#pragma unroll
        for (int e = 0; e + 3 < VEC; e += 4) {
            const floatx4 q = *(const floatx4*)(w + c + e);
            f[e] = q[0]; f[e + 1] = q[1]; f[e + 2] = q[2]; f[e + 3] = q[3];
        }
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = w[c + e];
    }
}

// values of the groups that channels c .. c + VEC - 1 belong to
template <int VEC>
__device__ __forceinline__ void norm_of_groups(const float* of, int c, int cg, float (&f)[VEC])
{
    int g = c / cg, rest = c - g * cg;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        f[e] = of[g];
        if (++rest == cg) { rest = 0; ++g; }
    }
}

template <class T, int VEC>
__device__ __forceinline__ Pack<T, VEC> norm_pack(const float (&f)[VEC])
{
    Pack<T, VEC> o;
#pragma unroll
    for (int e = 0; e < VEC; e += Pack<T, VEC>::SET) o.set(e, f + e);
    return o;
}

__device__ __forceinline__ double norm_block_sum(double v, double* scratch)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();                             // the previous sum's readers are done
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    return (scratch[0] + scratch[1]) + (scratch[2] + scratch[3]);
}

// One workgroup per row and group, three passes over memory; a wavefront's lanes along the group's channels.  A lane adds
// up to a 256th of a group of any length one by one: in 64 bits (in 32, the mean of 21 million values around 100 was off by
// 0.008; the time is the same, the loads').
template <class T>
__global__ __launch_bounds__(256) void norm_plain_kernel(NormArgs p)
{
    __shared__ double scratch[4];
    const int cg = p.C / p.G, g = blockIdx.x % p.G, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const size_t base = (blockIdx.x / p.G) * (size_t)p.P * p.C + (size_t)g * cg;
    const double count = (double)((size_t)p.P * cg);
    const T* x = (const T*)p.x + base;
    T* y = (T*)p.y + base;
    double s = 0.0;
    for (int i = wave; i < p.P; i += 4)
        for (int c = lane; c < cg; c += 64) s += (double)(float)x[(size_t)i * p.C + c];
    const float mean = (float)(norm_block_sum(s, scratch) / count);
    double m2 = 0.0;
    for (int i = wave; i < p.P; i += 4)
        for (int c = lane; c < cg; c += 64) {
            const double d = (float)x[(size_t)i * p.C + c] - mean;
            m2 = fma(d, d, m2);
        }
    const float rstd = 1.0f / sqrtf((float)(norm_block_sum(m2, scratch) / count) + p.eps);
    for (int i = wave; i < p.P; i += 4)
        for (int c = lane; c < cg; c += 64) {
            const int ch = g * cg + c;
            y[(size_t)i * p.C + c] = (T)norm_finish<T>((float)x[(size_t)i * p.C + c] - mean, p.weight ? rstd * p.weight[ch] : rstd, p.bias ? p.bias[ch] : 0.0f, p.act);
        }
}

// points == 1: L lanes own a group of cg = up to L * E * VEC channels, E vectors a lane.
constexpr int NORM_SEGMENT_THREADS = 256;
template <class T, int VEC, int E>
__global__ __launch_bounds__(NORM_SEGMENT_THREADS) void norm_segment_kernel(NormArgs p, int log_lanes, uint32_t segments)
{
    const int L = 1 << log_lanes, cg = p.C / p.G, sub = threadIdx.x & (L - 1);
    const uint32_t seg = blockIdx.x * (NORM_SEGMENT_THREADS >> log_lanes) + (threadIdx.x >> log_lanes);
    if (seg >= segments) return;                             // (all lanes of a group together)
    const int ch0 = (int)(seg % (uint32_t)p.G) * cg;
    const T* x = (const T*)p.x + (size_t)seg * cg;
    Pack<T, VEC> d[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int c = (sub + i * L) * VEC;
        if (c < cg) d[i] = *(const Pack<T, VEC>*)(x + c);
    }
    float w[E][VEC], b[E][VEC], s = 0.0f, m2 = 0.0f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int c = (sub + i * L) * VEC;
        if (c < cg) {
            norm_params<VEC>(p.weight, ch0 + c, p.vec_params, 1.0f, w[i]);
            norm_params<VEC>(p.bias, ch0 + c, p.vec_params, 0.0f, b[i]);
        }
    }
    const float inv = 1.0f / (float)cg;
#pragma unroll
    for (int i = 0; i < E; ++i)
        if ((sub + i * L) * VEC < cg)
#pragma unroll
            for (int e = 0; e < VEC; ++e) s += d[i].get(e);
    for (int off = L / 2; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
    const float mean = s * inv;
#pragma unroll
    for (int i = 0; i < E; ++i)
        if ((sub + i * L) * VEC < cg)
#pragma unroll
            for (int e = 0; e < VEC; ++e) { const float f = d[i].get(e) - mean; m2 = fmaf(f, f, m2); }
    for (int off = L / 2; off > 0; off >>= 1) m2 += __shfl_xor(m2, off, 64);
    const float rstd = 1.0f / sqrtf(m2 * inv + p.eps);
    T* y = (T*)p.y + (size_t)seg * cg;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int c = (sub + i * L) * VEC;
        if (c < cg) {
            float f[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = norm_finish<T>(d[i].get(e) - mean, rstd * w[i][e], b[i][e], p.act);
            *(Pack<T, VEC>*)(y + c) = norm_pack<T, VEC>(f);
        }
    }
}

// A workgroup's view of a slice of `cw` channels (whole groups) of some points: thread t owns vector column t % cols of
// points t / cols, + rows, ...: its channels never change.  Where the columns are a power of two up to 32, a wavefront
// first adds its points by shuffles.
struct NormTile {
    int cols, rows;              // vector columns; points per round
    int col, row;                // this thread's
    int cg, groups;              // channels a group, groups in the slice
    bool on, pow2;
    __device__ __forceinline__ NormTile(int cw, int cg_, int vec, int threads)
    {
        cols = cw / vec; rows = threads / cols; cg = cg_; groups = cw / cg_;
        row = (int)threadIdx.x / cols; col = (int)threadIdx.x - row * cols;
        on = row < rows;
        pow2 = cols <= 32 && (cols & (cols - 1)) == 0;
    }
    // this thread's first vector, in bytes (a round is at most 1024 points of less than 2^20 bytes each: norm_plan)
    template <int VEC> __device__ __forceinline__ uint32_t offset(size_t C, size_t size) const { return (uint32_t)(((size_t)row * C + col * VEC) * size); }
};

// Sums of every group of the slice from each thread's sums per channel (s[e], zero where the thread has nothing), into
// out[groups].  part: VEC * threads floats.  All threads call; two barriers.
template <int VEC, int NT>
__device__ __forceinline__ void norm_group_sums(const NormTile& t, float (&s)[VEC], float* part, float* out)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // channels of one group that a thread holds side by side are added at once
    int slots, m;                                            // partial sums a thread leaves; columns (or channels) a group spans
    if (t.cg % VEC == 0) {
#pragma unroll
        for (int e = 1; e < VEC; ++e) s[0] += s[e];
        slots = 1; m = t.cg / VEC;
    } else if (VEC % t.cg == 0) {
        slots = VEC / t.cg; m = 1;
        if constexpr (VEC >= 8) if (t.cg == 4) {
#pragma unroll
            for (int e = 1; e < 4; ++e) { s[0] += s[e]; s[4] += s[4 + e]; }
            s[1] = s[4];
        }
        if constexpr (VEC >= 4) if (t.cg == 2) {
#pragma unroll
            for (int e = 0; e < VEC / 2; ++e) s[e] = s[2 * e] + s[2 * e + 1];
        }
    } else { slots = VEC; m = t.cg; }
    int rows = t.rows, at = t.row * t.cols + t.col;
    bool write = t.on;
    if (t.pow2) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) if (e < slots)
            for (int off = 32; off >= t.cols; off >>= 1) s[e] += __shfl_xor(s[e], off, 64);
        rows = NT / 64; at = wave * t.cols + t.col;
        write = lane < t.cols;
    }
    const int plane = rows * t.cols;
    __syncthreads();                                         // (the previous call's readers of part and out are done)
    if (write)
#pragma unroll
        for (int e = 0; e < VEC; ++e) if (e < slots) part[e * plane + at] = s[e];
    __syncthreads();
    const int n = rows * m;
    for (int g = wave; g < t.groups; g += NT / 64) {
        float v = 0.0f;
        for (int i = lane; i < n; i += 64) {
            const int r = m == 1 ? i : i / m, j = m == 1 ? 0 : i - r * m;
            if (slots == 1) v += part[r * t.cols + g * m + j];
            else if (slots < VEC || t.cg == 1) v += part[(g % slots) * plane + r * t.cols + g / slots];
            else { const int c = g * t.cg + j; v += part[(c % VEC) * plane + r * t.cols + c / VEC]; }
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
        if (lane == 0) out[g] = v;
    }
    __syncthreads();
}

// Up to E vectors a thread of the `points` points from x on.  The address is a base that all threads share, one per i,
// plus an offset of 32 bits that does not change: with an address of its own each, the loads and stores in flight take
// more registers than the values.
template <class T, int VEC, int E>
__device__ __forceinline__ void norm_tile_load(const NormTile& t, const T* x, size_t C, int points, Pack<T, VEC> (&d)[E])
{
    const uint32_t off = t.offset<VEC>(C, sizeof(T));
    const size_t step = (size_t)t.rows * C;
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (t.on && t.row + i * t.rows < points) d[i] = *(const Pack<T, VEC>*)((const char*)(x + i * step) + off);
}

// Mean and sum of squared differences of every group over `points` points that the threads hold: into mean[], m2[].
template <class T, int VEC, int NT, int E>
__device__ __forceinline__ void norm_tile_stats(const NormTile& t, int points, Pack<T, VEC> (&d)[E], float* part, float* mean, float* m2)
{
    float s[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) s[e] = 0.0f;
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (t.on && t.row + i * t.rows < points)
#pragma unroll
            for (int e = 0; e < VEC; ++e) s[e] += d[i].get(e);
    norm_group_sums<VEC, NT>(t, s, part, mean);
    const float inv = 1.0f / ((float)points * (float)t.cg);
    for (int g = threadIdx.x; g < t.groups; g += NT) mean[g] *= inv;
    __syncthreads();
    constexpr int H = VEC < 4 ? VEC : 4;                     // (four channels at a time: few means are live at once)
#pragma unroll
    for (int h = 0; h < VEC; h += H) {
        float mu[H];
        norm_of_groups<H>(mean, t.on ? t.col * VEC + h : 0, t.cg, mu);
#pragma unroll
        for (int e = 0; e < H; ++e) s[h + e] = 0.0f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            norm_keep_packed(d[i]);
            if (t.on && t.row + i * t.rows < points)
#pragma unroll
                for (int e = 0; e < H; ++e) { const float f = d[i].get(h + e) - mu[e]; s[h + e] = fmaf(f, f, s[h + e]); }
        }
    }
    norm_group_sums<VEC, NT>(t, s, part, m2);
}

// One workgroup per row and slice of cw channels, everything it owns in registers.  The second bound, 64 registers a lane,
// lets two workgroups of 1024 threads share a compute unit; the forms of 7 and 8 vectors of 8 bf16 pass it by 3 and 10
// registers, which go through scratch.  The form of 7 is taken where 7 vectors a thread hold the row: it keeps most of them
// (1024 rows of 36 x 48 points of 32 bf16: 56.8 us, in the form of 8 65.7).
template <class T, int VEC, int NT, int E>
__global__ __launch_bounds__(NT, 8) void norm_resident_kernel(NormArgs p, int cw)
{
    extern __shared__ float norm_lds[];
    const int cg = p.C / p.G;
    const uint32_t slices = p.C / cw;
    const NormTile t(cw, cg, VEC, NT);
    float* part = norm_lds;
    float* mean = part + VEC * NT;
    float* m2 = mean + t.groups;
    const int c0 = (int)(blockIdx.x % slices) * cw;
    const size_t base = blockIdx.x / slices * ((size_t)p.P * p.C) + c0;
    Pack<T, VEC> d[E];
    norm_tile_load<T, VEC, E>(t, (const T*)p.x + base, p.C, p.P, d);
    norm_tile_stats<T, VEC, NT, E>(t, p.P, d, part, mean, m2);
    for (int g = threadIdx.x; g < t.groups; g += NT) m2[g] = 1.0f / sqrtf(m2[g] / ((float)p.P * (float)cg) + p.eps);
    __syncthreads();
    if (!t.on) return;
    // four channels of every vector at a time, the results in their place: few parameters are live at once
    constexpr int H = VEC < 4 ? VEC : 4;
#pragma unroll
    for (int h = 0; h < VEC; h += H) {
        const int c = t.col * VEC + h;
        float mu[H], r[H], w[H], b[H];
        norm_of_groups<H>(mean, c, cg, mu);
        norm_of_groups<H>(m2, c, cg, r);
        norm_params<H>(p.weight, c0 + c, p.vec_params, 1.0f, w);
        norm_params<H>(p.bias, c0 + c, p.vec_params, 0.0f, b);
#pragma unroll
        for (int e = 0; e < H; ++e) r[e] *= w[e];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            norm_keep_packed(d[i]);
            float f[H];
#pragma unroll
            for (int e = 0; e < H; ++e) f[e] = norm_finish<T>(d[i].get(h + e) - mu[e], r[e], b[e], p.act);
#pragma unroll
            for (int e = 0; e < H; e += Pack<T, VEC>::SET) d[i].set(h + e, f + e);
        }
    }
    T* y = (T*)p.y + base;
    const uint32_t off = t.offset<VEC>(p.C, sizeof(T));
    const size_t step = (size_t)t.rows * p.C;
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (t.row + i * t.rows < p.P) *(Pack<T, VEC>*)((char*)(y + i * step) + off) = d[i];
}

// (count, mean, sum of squared differences) of two disjoint sets, joined.
__device__ __forceinline__ void norm_join(float& n, float& mean, float& m2, float nb, float meanb, float m2b)
{
    const float total = n + nb;
    if (nb > 0.0f) {
        const float d = meanb - mean, f = nb / total;
        mean = fmaf(d, f, mean);
        m2 += fmaf(d * (n * f), d, m2b);         // (in this order zero weights come before what may overflow)
        n = total;
    }
}

// Split, first kernel: a workgroup per row, slice and run of points; stats[row][group][run] = (mean, sum of squared
// differences) of the run.  A thread joins its channels' values batch by batch, each batch held in registers for its two
// passes, the next one on its way; the threads meet once, at the run's end: with two sums over the workgroup for every
// batch, their barriers left the memory idle (83 MB read, as many written back: 37 us so, 31 us now, the same for 4 or 8 points
// a batch and 512 or 1024 workgroups).
constexpr int NORM_SPLIT_THREADS = 512, NORM_SPLIT_U = 4, NORM_APPLY_THREADS = 1024;
template <class T, int VEC>
__global__ __launch_bounds__(NORM_SPLIT_THREADS) void norm_stats_kernel(NormArgs p, int cw, int runs, int run_points, float2* stats)
{
    constexpr int NT = NORM_SPLIT_THREADS, U = NORM_SPLIT_U;
    extern __shared__ float norm_lds[];
    const int cg = p.C / p.G, slices = p.C / cw;
    const NormTile t(cw, cg, VEC, NT);
    float* part = norm_lds;
    float* mean = part + VEC * NT;
    float* m2 = mean + t.groups;
    const int slice = (int)(blockIdx.x % slices), run = (int)(blockIdx.x / slices % runs);
    const size_t n = blockIdx.x / slices / runs;
    // (points are counted in 32 bits without a sign: a round past the last one of 2^31 - 1 stays below 2^32)
    const uint32_t first = (uint32_t)run * run_points, last = min((uint32_t)p.P, first + run_points), tile = t.rows * U;
    const T* x = (const T*)p.x + n * (size_t)p.P * p.C + slice * cw;
    Pack<T, VEC> d[U], next[U];
    float mu[VEC], sq[VEC], have = 0.0f;                     // of this thread's channels, over `have` points
#pragma unroll
    for (int e = 0; e < VEC; ++e) mu[e] = sq[e] = 0.0f;
    norm_tile_load<T, VEC, U>(t, x + (size_t)first * p.C, p.C, (int)(last - first), d);
    for (uint32_t at = first; at < last; at += tile) {
        if (at + tile < last) norm_tile_load<T, VEC, U>(t, x + (size_t)(at + tile) * p.C, p.C, (int)(last - at - tile), next);
        const int left = t.on ? (int)(last - at) - t.row : 0;       // (u * rows < left: there is a point)
        if (left > 0) {
            const float batch = (float)min(U, (left + t.rows - 1) / t.rows), total = have + batch, f = batch / total, inv = 1.0f / batch;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                float s = 0.0f, q = 0.0f;
#pragma unroll
                for (int u = 0; u < U; ++u) s += u * t.rows < left ? d[u].get(e) : 0.0f;
                s *= inv;
#pragma unroll
                for (int u = 0; u < U; ++u) { const float g = u * t.rows < left ? d[u].get(e) - s : 0.0f; q = fmaf(g, g, q); }
                const float g = s - mu[e];
                mu[e] = fmaf(g, f, mu[e]);
                sq[e] += fmaf(g * (have * f), g, q);
            }
            have = total;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) d[u] = next[u];
    }
    float s[VEC], of[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) s[e] = mu[e] * have;
    norm_group_sums<VEC, NT>(t, s, part, mean);
    const float inv = 1.0f / ((float)(last - first) * (float)cg);
    for (int g = threadIdx.x; g < t.groups; g += NT) mean[g] *= inv;
    __syncthreads();
    norm_of_groups<VEC>(mean, t.on ? t.col * VEC : 0, cg, of);
#pragma unroll
    for (int e = 0; e < VEC; ++e) { const float g = mu[e] - of[e]; s[e] = have > 0.0f ? fmaf(g * have, g, sq[e]) : 0.0f; }
    norm_group_sums<VEC, NT>(t, s, part, m2);
    for (int g = threadIdx.x; g < t.groups; g += NT)
        stats[(n * p.G + slice * t.groups + g) * runs + run] = make_float2(mean[g], m2[g]);
}

// Split, second kernel: every workgroup joins the runs of its row (a wavefront per group, lanes over runs, always in the
// same order) and writes its points.
template <class T, int VEC>
__global__ __launch_bounds__(NORM_APPLY_THREADS) void norm_apply_kernel(NormArgs p, int cw, int runs, int run_points, const float2* stats, int parts, int part_points)
{
    extern __shared__ float norm_lds[];
    const int cg = p.C / p.G, slices = p.C / cw, lane = threadIdx.x & 63;
    const NormTile t(cw, cg, VEC, NORM_APPLY_THREADS);
    float* mean = norm_lds;
    float* rstd = mean + t.groups;
    const int slice = (int)(blockIdx.x % slices), piece = (int)(blockIdx.x / slices % parts);
    const size_t n = blockIdx.x / slices / parts;
    for (int g = threadIdx.x >> 6; g < t.groups; g += NORM_APPLY_THREADS / 64) {
        float cnt = 0.0f, a = 0.0f, b = 0.0f;
        for (int r = lane; r < runs; r += 64) {
            const float2 s = stats[(n * p.G + slice * t.groups + g) * runs + r];
            norm_join(cnt, a, b, (float)min(run_points, p.P - r * run_points) * (float)cg, s.x, s.y);
        }
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const float cb = __shfl_xor(cnt, off, 64), ab = __shfl_xor(a, off, 64), bb = __shfl_xor(b, off, 64);
            // (the lower lane's set first: both lanes of a pair get the same bits)
            if (lane & off) { float c2 = cb, a2 = ab, b2 = bb; norm_join(c2, a2, b2, cnt, a, b); cnt = c2; a = a2; b = b2; }
            else norm_join(cnt, a, b, cb, ab, bb);
        }
        if (lane == 0) { mean[g] = a; rstd[g] = 1.0f / sqrtf(b / cnt + p.eps); }
    }
    __syncthreads();
    if (!t.on) return;
    const int c0 = slice * cw;
    float mu[VEC], r[VEC], w[VEC], b[VEC];
    norm_of_groups<VEC>(mean, t.col * VEC, cg, mu);
    norm_of_groups<VEC>(rstd, t.col * VEC, cg, r);
    norm_params<VEC>(p.weight, c0 + t.col * VEC, p.vec_params, 1.0f, w);
    norm_params<VEC>(p.bias, c0 + t.col * VEC, p.vec_params, 0.0f, b);
#pragma unroll
    for (int e = 0; e < VEC; ++e) r[e] *= w[e];
    const size_t base = n * (size_t)p.P * p.C + c0, step = (size_t)t.rows * p.C;
    const uint32_t off = t.offset<VEC>(p.C, sizeof(T));
    const uint32_t begin = (uint32_t)piece * part_points, last = min((uint32_t)p.P, begin + part_points);
    constexpr int U = 2;                                     // loads in flight
    for (uint32_t first = begin; first < last; first += U * t.rows) {
        const uint32_t at = first + t.row;
        const T* x = (const T*)p.x + base + (size_t)first * p.C;
        T* y = (T*)p.y + base + (size_t)first * p.C;
        Pack<T, VEC> d[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (at + u * t.rows < last) d[u] = *(const Pack<T, VEC>*)((const char*)(x + u * step) + off);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (at + u * t.rows < last) {
                float f[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[e] = norm_finish<T>(d[u].get(e) - mu[e], r[e], b[e], p.act);
                *(Pack<T, VEC>*)((char*)(y + u * step) + off) = norm_pack<T, VEC>(f);
            }
    }
}

// How a call is laid out; from sizes and alignment alone.
enum NormKind { NORM_SEGMENT, NORM_RESIDENT, NORM_SPLIT, NORM_PLAIN };
struct NormPlan {
    NormKind kind;
    int vec;                     // elements a vector
    int lanes, per_lane;         // segment: lanes a group, vectors a lane
    int cw, threads;             // resident, split: channels a slice; resident: threads
    int runs, run_points, parts, part_points;      // split
    size_t workspace;
};

// vec: elements a 16-byte (or smaller) access may take, as far as the addresses go.
static inline NormPlan norm_plan(int N, int P, int C, int G, int size, int vec)
{
    NormPlan q{};
    const int cg = C / G;
    // a vector never leaves a row's channels
    while (C % vec) vec /= 2;
    q.vec = vec;
    const bool wide = (int64_t)C * size >= (int64_t)1 << 20;         // (a round's offsets would leave 32 bits)
    if (P == 1) {
        int v = vec;
        while (cg % v) v /= 2;
        const int n = cg / v;
        int lanes = 1;
        while (lanes * 2 < n && lanes < 64) lanes *= 2;          // (two vectors a lane: 33.5 MB in 65536 groups of 128, bf16: 9.4 us; one: 10.1, four: 10.7)
        if (n <= lanes * 8) {
            q.kind = NORM_SEGMENT; q.vec = v; q.lanes = lanes; q.per_lane = (n + lanes - 1) / lanes;
            return q;
        }
    }
    // Slices of whole groups and whole vectors.  A slice's points are runs of cw * size bytes; below 128 bytes they no
    // longer fill a line of the cache, so smaller slices are taken only if the channels are no more.
    const int unit = std::lcm(cg, vec);
    auto fits = [&](int cw, int threads, int e) { return cw / vec <= threads && cw / cg <= 2048 && ((int64_t)P + threads / (cw / vec) - 1) / (threads / (cw / vec)) <= e; };
    int best = 0, widest = 0;
    for (int k = 1; k <= C / unit && !(wide && P > 1); ++k) {
        const int cw = unit * k;
        if (cw / vec > 1024 || cw / cg > 2048) break;
        if (C % cw) continue;
        if (cw * size < 128 && cw != C) continue;
        // split: two points a round where there are such slices, else one (4 rows of 1728 points of 1280 fp32 channels in one
        // group, 320 vectors: 27 us; by the plain kernel 8.7 ms)
        if (cw / vec <= NORM_SPLIT_THREADS / 2 || (!widest && cw / vec <= NORM_SPLIT_THREADS)) widest = cw;
        // the widest slice that fits, but narrower ones while the rows alone leave compute units without work
        if (fits(cw, 1024, 8) && (!best || (int64_t)N * (C / cw) >= 256)) best = cw;
    }
    if (best && C / best <= 1 << 20) {                       // (a row's workgroups fit a launch)
        q.kind = NORM_RESIDENT; q.cw = best;
        q.threads = fits(best, 256, 4) ? 256 : fits(best, 512, 8) ? 512 : 1024;
        return q;
    }
    if (!widest || P == 1) { q.kind = NORM_PLAIN; return q; }
    q.kind = NORM_SPLIT; q.cw = widest;
    // about 512 workgroups (two a compute unit) of at least a batch, at most 256 a row (every workgroup of the second
    // kernel reads them all)
    const int tile = NORM_SPLIT_THREADS / (widest / vec) * NORM_SPLIT_U;
    const int64_t want = std::max<int64_t>(1, 512 / std::max<int64_t>(1, (int64_t)N * (C / widest)));
    const int64_t runs = std::min<int64_t>(std::min<int64_t>(want, 256), ((int64_t)P + tile - 1) / tile);
    q.run_points = (int)((P + runs - 1) / runs);
    q.runs = (int)(((int64_t)P + q.run_points - 1) / q.run_points);
    // second kernel: 512 workgroups of 1024 threads (83 MB read and written: 34 us; 1024 of 512 threads: 40 us)
    const int64_t pieces = std::max<int64_t>(1, std::min<int64_t>(512 / std::max<int64_t>(1, (int64_t)N * (C / widest)), ((int64_t)P + 31) / 32));
    q.part_points = (int)((P + pieces - 1) / pieces);
    q.parts = (int)(((int64_t)P + q.part_points - 1) / q.part_points);
    q.workspace = (size_t)N * q.runs * G * sizeof(float2);
    return q;
}

template <class T, int VEC>
static void norm_launch_vec(const NormArgs& p, const NormPlan& q, void* workspace, hipStream_t s)
{
    const int cg = p.C / p.G;
    if (q.kind == NORM_SEGMENT) {
        const uint32_t segments = (uint32_t)((size_t)p.N * p.G), per = NORM_SEGMENT_THREADS / q.lanes;
        const int log_lanes = __builtin_ctz(q.lanes);
        auto go = [&](auto e) {
            hipLaunchKernelGGL((norm_segment_kernel<T, VEC, decltype(e)::value>), dim3((segments + per - 1) / per), dim3(NORM_SEGMENT_THREADS), 0, s, p, log_lanes, segments);
        };
        using I1 = std::integral_constant<int, 1>; using I2 = std::integral_constant<int, 2>; using I4 = std::integral_constant<int, 4>; using I8 = std::integral_constant<int, 8>;
        if (q.per_lane == 1) go(I1{});
        else if (q.per_lane == 2) go(I2{});
        else if (q.per_lane <= 4) go(I4{});
        else go(I8{});
        return;
    }
    // at most 2^21 workgroups a launch (a grid's threads stay below 2^32); runs and parts are more than one only where
    // rows and slices are few.  (slices are at most 2^20: norm_plan, and 2^20 / 128 where points > 1)
    const int slices = p.C / q.cw, groups = q.cw / cg, most = (1 << 21) / slices;
    for (int first = 0; first < p.N; first += most) {
        NormArgs a = p;
        a.N = std::min(most, p.N - first);
        a.x = (const T*)p.x + (size_t)first * p.P * p.C;
        a.y = (T*)p.y + (size_t)first * p.P * p.C;
        const unsigned blocks = (unsigned)a.N * slices;
        if (q.kind == NORM_RESIDENT) {
            const size_t lds = (size_t)(VEC * q.threads + 2 * groups) * sizeof(float);
            const int rows = q.threads / (q.cw / VEC), e = (p.P + rows - 1) / rows;
            auto go = [&](auto nt, auto ee) {
                constexpr int NT = decltype(nt)::value, E = decltype(ee)::value;
                hipLaunchKernelGGL((norm_resident_kernel<T, VEC, NT, E>), dim3(blocks), dim3(NT), lds, s, a, q.cw);
            };
            using I2 = std::integral_constant<int, 2>; using I4 = std::integral_constant<int, 4>; using I8 = std::integral_constant<int, 8>;
            if (q.threads == 256) { if (e <= 2) go(std::integral_constant<int, 256>{}, I2{}); else go(std::integral_constant<int, 256>{}, I4{}); }
            else if (q.threads == 512) go(std::integral_constant<int, 512>{}, I8{});
            else if (e <= 7) go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 7>{});
            else go(std::integral_constant<int, 1024>{}, I8{});
        } else {
            float2* stats = (float2*)workspace + (size_t)first * q.runs * p.G;
            hipLaunchKernelGGL((norm_stats_kernel<T, VEC>), dim3(blocks * q.runs), dim3(NORM_SPLIT_THREADS),
                               (size_t)(VEC * NORM_SPLIT_THREADS + 2 * groups) * sizeof(float), s, a, q.cw, q.runs, q.run_points, stats);
            hipLaunchKernelGGL((norm_apply_kernel<T, VEC>), dim3(blocks * q.parts), dim3(NORM_APPLY_THREADS), (size_t)2 * groups * sizeof(float), s,
                               a, q.cw, q.runs, q.run_points, (const float2*)stats, q.parts, q.part_points);
        }
    }
}

template <class T>
static void norm_launch(const NormArgs& p, const NormPlan& q, void* workspace, hipStream_t s)
{
    if (q.kind == NORM_PLAIN) {
        hipLaunchKernelGGL((norm_plain_kernel<T>), dim3((unsigned)((size_t)p.N * p.G)), dim3(256), 0, s, p);
        return;
    }
    if constexpr (sizeof(T) == 2) if (q.vec == 8) return norm_launch_vec<T, 8>(p, q, workspace, s);
    if (q.vec == 4) norm_launch_vec<T, 4>(p, q, workspace, s);
    else if (q.vec == 2) norm_launch_vec<T, 2>(p, q, workspace, s);
    else norm_launch_vec<T, 1>(p, q, workspace, s);
}

}  // namespace seedinf
