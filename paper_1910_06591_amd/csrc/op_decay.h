// Linear attention with a decay for each head: a recurrent core whose state is a matrix per head,
//   S_t = g S_{t-1} + k_t v_t^T   (S_{t-1} taken as zero where done_t is set),    o_t = scale q_t^T S_t.
#pragma once
#include "op_common.h"

namespace seedinf {

struct DecayArgs {
    const void* q; const void* k; const void* v;
    const float* decay;          // [heads]
    const uint8_t* done;         // [steps, rows] or nullptr
    const int32_t* lengths;      // [rows] or nullptr
    const float* s_in;           // [rows, heads, dk, dv] or nullptr (zero)
    void* out;
    float* s_out;
    int64_t q_t, q_b, k_t, k_b, v_t, v_b, o_t, o_b;       // strides of a step and of a row, in elements
    int T, B, H, KV, dk, dv;
    float scale;
    int vec_state;               // dv and the states' addresses allow 16-byte accesses
};

__device__ __forceinline__ int decay_length(const DecayArgs& p, int b)
{
    if (!p.lengths) return p.T;
    const int n = p.lengths[b];
    return n < 0 ? 0 : (n > p.T ? p.T : n);
}

// The recurrence step by step: one workgroup holds dk x 64 of a head's state in registers (a thread 4 columns of
// every 16th row) and walks the steps.  State columns are independent of one another, so a wider value is several
// workgroups.  A step's o is a sum over dk: 4 rows of a wavefront by shuffles, the 4 wavefronts through LDS.
constexpr int DECAY_COLS = 64;
template <class T, int DK>
__global__ __launch_bounds__(256) void decay_recurrent_kernel(DecayArgs p)
{
    constexpr int R = DK / 16;                              // rows of the state a thread holds
    __shared__ float sq[DK], sk[DK], sv[DECAY_COLS];
    __shared__ floatx4 part[4][16];
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, wave = tid >> 6;
    const int tiles = (p.dv + DECAY_COLS - 1) / DECAY_COLS;
    const int tile = blockIdx.x % tiles, bh = blockIdx.x / tiles, h = bh % p.H, b = bh / p.H;
    const int hk = h / (p.H / p.KV);
    const int c0 = tile * DECAY_COLS + 4 * tx;              // this thread's first column
    const int nc = p.dv - c0;                               // columns that are there
    const float g = p.decay[h];
    const int len = decay_length(p, b);
    const size_t base = (size_t)bh * p.dk * p.dv;
    floatx4 S[R];
    const bool fresh = !p.s_in || (p.done && len > 0 && p.done[b]);       // the state given is not read
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = ty + 16 * r;
        S[r] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (fresh || row >= p.dk) continue;
        const float* src = p.s_in + base + (size_t)row * p.dv + c0;
        if (p.vec_state && nc >= 4) S[r] = *(const floatx4*)src;
        else
#pragma unroll
            for (int j = 0; j < 4; ++j) if (j < nc) S[r][j] = src[j];
    }
    const T* q = (const T*)p.q + (int64_t)b * p.q_b + (int64_t)h * p.dk;
    const T* k = (const T*)p.k + (int64_t)b * p.k_b + (int64_t)hk * p.dk;
    const T* v = (const T*)p.v + (int64_t)b * p.v_b + (int64_t)hk * p.dv;
    T* o = (T*)p.out + (int64_t)b * p.o_b + (int64_t)h * p.dv;
    for (int t = 0; t < len; ++t) {
        if (tid < DK) {
            sq[tid] = tid < p.dk ? (float)q[t * p.q_t + tid] * p.scale : 0.0f;
            sk[tid] = tid < p.dk ? (float)k[t * p.k_t + tid] : 0.0f;
        }
        if (tid < DECAY_COLS) sv[tid] = tile * DECAY_COLS + tid < p.dv ? (float)v[t * p.v_t + tile * DECAY_COLS + tid] : 0.0f;
        const bool reset = t > 0 && p.done && p.done[(int64_t)t * p.B + b];
        __syncthreads();
        const floatx4 vv = *(const floatx4*)&sv[4 * tx];
        floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float kr = sk[ty + 16 * r], qr = sq[ty + 16 * r];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                S[r][j] = fmaf(kr, vv[j], reset ? 0.0f : g * S[r][j]);
                acc[j] = fmaf(qr, S[r][j], acc[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            acc[j] += __shfl_xor(acc[j], 16, 64);
            acc[j] += __shfl_xor(acc[j], 32, 64);
        }
        if ((tid & 63) < 16) part[wave][tx] = acc;
        __syncthreads();
        if (tid < DECAY_COLS && tile * DECAY_COLS + tid < p.dv) {
            const float* f = (const float*)part;
            o[t * p.o_t + tile * DECAY_COLS + tid] = (T)((f[tid] + f[64 + tid]) + (f[128 + tid] + f[192 + tid]));
        }
        // (the next step's first barrier stands between these reads and the next writes of `part`; sq, sk and sv are
        // written before it, after this step's last read of them)
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = ty + 16 * r;
        if (row >= p.dk) continue;
        float* dst = p.s_out + base + (size_t)row * p.dv + c0;
        if (p.vec_state && nc >= 4) *(floatx4*)dst = S[r];
        else
#pragma unroll
            for (int j = 0; j < 4; ++j) if (j < nc) dst[j] = S[r][j];
    }
}

template <class T>
static void decay_launch(const DecayArgs& p, hipStream_t s)
{
    const unsigned grid = (unsigned)((size_t)p.B * p.H * ((p.dv + DECAY_COLS - 1) / DECAY_COLS));
    if (p.dk <= 64) hipLaunchKernelGGL((decay_recurrent_kernel<T, 64>), dim3(grid), dim3(256), 0, s, p);
    else if (p.dk <= 128) hipLaunchKernelGGL((decay_recurrent_kernel<T, 128>), dim3(grid), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((decay_recurrent_kernel<T, 256>), dim3(grid), dim3(256), 0, s, p);
}

}  // namespace seedinf
