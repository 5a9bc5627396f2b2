// Linear attention with a decay for each head: a recurrent core whose state is a matrix per head,
//   S_t = g S_{t-1} + k_t v_t^T   (S_{t-1} taken as zero where done_t is set),    o_t = scale q_t^T S_t.
#pragma once
#include <atomic>
#include <type_traits>

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
    int vec_in;                  // q, k and v: every head is 16-byte aligned and whole 16 bytes, a step's stride is below 2^25 bytes
    int vec_o;                   // 16 bytes of outputs can be stored at once
    int segments, segment_steps; // the time axis in parts that are worked on side by side; 1: not split
    float* seg_state;            // [rows, heads, segments, dk, dv]: what a segment adds to the state, then the state in front of it
    float2* seg_factor;          // [rows, heads, segments]: (power of the decay over the segment, 1 if a flag lies in it)
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
// Bound by the state, read and written once: one step of 256 rows, 16 heads of 128 x 128 (537 MB) 101 us, 5.3 TB/s,
// what a large copy reaches; 8 rows of 4 heads of 64 x 64 4.2 us, a launch's own time.
// The wavefronts a SIMD are asked for: left alone, the compiler takes twice the registers for 128 rows, and that step 115 us.
constexpr int DECAY_COLS = 64;
template <class T, int DK>
__global__ __launch_bounds__(256, DK == 64 ? 8 : DK == 128 ? 6 : 4) void decay_recurrent_kernel(DecayArgs p)
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
        // Rows behind key_dim are zero, but 0 times an infinite value is NaN: then they are cleared, and the sums made anew.
        if (const floatx4 zero = vv * 0.0f; p.dk < DK && !(zero[0] + zero[1] + zero[2] + zero[3] == 0.0f)) {
            int row = ty;
            asm volatile("" : "+v"(row));                   // (the rows' conditions are not kept in registers from the loads on)
            acc = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int r = 0; r < R; ++r, row += 16) {
                if (row >= p.dk) S[r] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] = fmaf(sq[row], S[r][j], acc[j]);
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

// ---- chunks: matrix products over 64 steps (bf16) or 32 (fp32) ----
//
// With S the state in front of a chunk, steps i, j counted inside it, and no flags,
//   o_i = scale (g^(i+1) q_i^T S + sum_{j <= i} g^(i-j) (q_i . k_j) v_j),   S' = g^c S + sum_j g^(c-1-j) k_j v_j^T,
// four products on the matrix units: scores, scores x values, queries x state, keys^T x values.  A flag at step r cuts
// every power that spans it: j >= r where i >= r, and S takes no part from r on.  Powers are a table (in 64 bits, by
// squaring: no logarithm of a decay of 0 or 1), never negative: nothing overflows where a decay is small.
//
// A workgroup (4 wavefronts) owns up to 128 columns of a head's state, each wavefront a quarter of the columns and all
// rows, in accumulator registers for the whole time axis: S never travels through LDS.  The rows of the accumulator
// tiles are the state's in an order (decay_row) in which a lane's values of two tiles are the eight consecutive key
// elements that a bf16 operand wants, so S is an operand as it stands.
//
// Roundings: bf16 inputs are operands as they are.  What is computed between the products (scores, the state as an operand,
// the weighted values of its update) is fp32 and is split into three bf16 parts whose sum it is, 24 bits, so that nothing
// is lost (in two parts outputs were 1.0e-4 of their norm off, and the split axes below 10 % faster).  fp32 inputs use the
// fp32 matrix instructions.
//
// What bounds it: 32768 steps of 16 heads of 128 x 128, bf16, are 537 MB (85 us) and, with the parts, 16 MFLOP a chunk for
// outputs and 6 for the segments' states, 183 GFLOP (150 us at a large matrix product's rate); and a chunk's phases, each of
// which waits for the one before it: LDS writes of keys and values with their steps side by side, scores, their split, the
// products with the state in accumulators.  Two workgroups a compute unit fill one another's gaps as far as registers (256
// a lane) and LDS (80 KiB) allow.  Split into 32 segments: what they add to the state 85 us, the scan of the states 20, the
// outputs 171; 4 prompts of up to 4001 steps in 8 segments: 37 + 18 + 80; fp32, 32 steps of 128 rows of 4 heads of 64 x 64,
// not split: 12.9 us of which the state's 16.8 MB take 3; it goes in and out of accumulators in accesses of 4 bytes.
//
// From a chunk on in which a key, a value, a score or a query times the state is not finite, a workgroup walks its steps as
// the recurrence says, on the state in memory.  The products would carry such a value into steps before it and past flags
// (zero times infinity), the parts of an infinity are an infinity and NaN, and a score is a product that the recurrence never
// forms: of a large query with a later key, too.  What is not finite in queries and in the state shows in their products.
// (It does not come back to chunks: with the state in accumulators on both sides of a
// walk, 32768 steps of 16 heads of 128 x 128 took 281 us in place of 271.)

template <class T> struct DecayMma;
template <> struct DecayMma<float> {
    static constexpr int C = 32, FE = 4, KS = 16;           // steps a chunk; elements of an operand a lane; depth of a product
    typedef floatx4 Frag;
    static __device__ __forceinline__ floatx4 mma(floatx4 a, floatx4 b, floatx4 c)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};
template <> struct DecayMma<__bf16> {
    static constexpr int C = 64, FE = 8, KS = 32;
    typedef bf16x8 Frag;
    static __device__ __forceinline__ floatx4 mma(bf16x8 a, bf16x8 b, floatx4 c) { return mfma16(a, b, c); }
};

// the state's row that row m of accumulator tile t holds
template <class T> __device__ __forceinline__ int decay_row(int t, int m)
{
    if constexpr (sizeof(T) == 4) return 16 * t + m;
    else return 32 * (t >> 1) + 8 * (m >> 2) + 4 * (t & 1) + (m & 3);
}

__device__ __forceinline__ bf16x8 decay_round8(const float (&x)[8]) { return to_bf16x8(floatx4{x[0], x[1], x[2], x[3]}, floatx4{x[4], x[5], x[6], x[7]}); }
// x = hi + rest: rest in place of x
__device__ __forceinline__ bf16x8 decay_split8(float (&x)[8])
{
    const bf16x8 hi = decay_round8(x);
    const u32x4 w = __builtin_bit_cast(u32x4, hi);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[2 * e] -= bf16_lo_f32(u[e]); x[2 * e + 1] -= bf16_hi_f32(u[e]); }
    return hi;
}

// FE elements of a row of `dim` elements from element d on, one by one, zero behind its end
template <class T>
__device__ __forceinline__ u32x4 decay_load16(const T* row, int d, int dim)
{
    constexpr int FE = DecayMma<T>::FE;
    union { u32x4 u; T e[FE]; } x;
    x.u = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < FE; ++i) if (d + i < dim) x.e[i] = row[d + i];
    return x.u;
}

// the largest magnitude's bits, per element: an exponent of all ones is a value that is not finite
template <class T>
__device__ __forceinline__ uint32_t decay_magnitude(uint32_t seen, uint32_t w)
{
    if constexpr (sizeof(T) == 4) { const uint32_t m = w & 0x7fffffffu; return m > seen ? m : seen; }
    else {
        typedef unsigned short ushortx2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushortx2, seen), __builtin_bit_cast(ushortx2, w & 0x7fff7fffu)));
    }
}
template <class T>
__device__ __forceinline__ bool decay_not_finite(uint32_t seen)
{
    if constexpr (sizeof(T) == 4) return seen >= 0x7f800000u;
    else return (seen & 0xffffu) >= 0x7f80u || (seen >> 16) >= 0x7f80u;
}

// LDS rows of R bytes without padding; 16-byte pieces of a 256-byte line change places with the row, so that the 16
// rows (lanes) and 4 pieces (lane groups) of an operand read fall on different banks.
template <int R> __device__ __forceinline__ uint32_t decay_at(int row, int piece)
{
    if constexpr (R == 128) return (uint32_t)((row >> 1) * 256 + ((((row & 1) << 3) | piece) ^ ((row >> 1) & 7)) * 16);
    else return (uint32_t)(row * R + ((piece & ~15) | ((piece ^ row) & 15)) * 16);
}
// The operand of rows 16 t + ln and pieces 4 ks + lg: `x` is decay_operand_x<R>(ln, lg); t and ks are constants.
template <int R> __device__ __forceinline__ uint32_t decay_operand_x(int ln, int lg) { return decay_at<R>(ln, lg); }
template <int R> __device__ __forceinline__ uint32_t decay_operand(uint32_t x, int t, int ks)
{
    if constexpr (R == 128) return (x ^ (uint32_t)(ks * 64)) + (uint32_t)(t * 16 * R);
    else return (x ^ (uint32_t)((ks & 3) * 64)) + (uint32_t)(t * 16 * R + (ks >> 2) * 256);
}

template <class T, int DK, int DVT, bool OUT> struct DecayLds {
    static constexpr int C = DecayMma<T>::C;
    static constexpr int KROW = DK * (int)sizeof(T), CROW = C * (int)sizeof(T), PARTS = sizeof(T) == 4 ? 1 : 3;      // bytes a row
    static constexpr int NQ = OUT ? C * KROW : 0, NK = OUT ? (KROW > PARTS * CROW ? C * KROW : PARTS * C * CROW) : 0;
    // queries; keys, later the scores' parts; keys and values with their steps side by side; tables
    static constexpr int Q = 0, K = NQ, KT = K + NK, VT = KT + DK * CROW, END = VT + DVT * CROW;
    static constexpr size_t BYTES = (size_t)END + (2 * C + 8) * sizeof(float) + 32 + (OUT ? (C + 4 + 512) * sizeof(float) : 0);
    static constexpr int RESIDENT = BYTES <= 80 * 1024 ? 2 : 1;          // workgroups a compute unit
};

// the row of the transposed arrays that element d stands in: the order of the accumulators' rows (decay_row's inverse)
template <class T> __device__ __forceinline__ int decay_place(int d)
{
    if constexpr (sizeof(T) == 4) return d;
    else return (d & ~31) | ((d & 4) << 2) | ((d & 24) >> 1) | (d & 3);
}

// Steps t0 .. stop as the recurrence says, on the state of DVT columns in memory: a thread has a column and R of its rows.
// Returns the power of the decay over them, and 1 if a flag lies among them.
template <class T, int DK, int DVT, bool OUT>
__device__ __forceinline__ float2 decay_walk(char* lds, const T* q, const T* k, const T* v, T* o, float* state, const uint8_t* done, float g, float scale,
                                             int64_t q_t, int64_t k_t, int64_t v_t, int64_t o_t, int B, int dk, int dv, int dvt, int t0, int stop)
{
    constexpr int RG = 256 / DVT, R = DK / RG;
    float* const key = (float*)lds; float* const query = key + DK; float* const part = query + DK;
    const int tid = threadIdx.x, col = tid % DVT, row0 = tid / DVT * R;
    const bool on = col < dvt;
    __syncthreads();                                         // (the state is there, and what LDS holds is read)
    float x[R], factor = 1.0f, cut = 0.0f;
#pragma unroll
    for (int i = 0; i < R; ++i) x[i] = on && row0 + i < dk ? state[(size_t)(row0 + i) * dv + col] : 0.0f;
    float next_k = 0.0f, next_q = 0.0f, next_v = 0.0f;       // a step's elements, on their way while the one before it is worked on
    bool next_reset = false;
    auto fetch = [&](int t) {
        if (tid < dk) {
            next_k = (float)k[(int64_t)t * k_t + tid];
            if (OUT) next_q = (float)q[(int64_t)t * q_t + tid];
        }
        if (on) next_v = (float)v[(int64_t)t * v_t + col];
        next_reset = done && done[(int64_t)t * B];
    };
    fetch(t0);
    for (int t = t0; t < stop; ++t) {
        const bool reset = next_reset;
        const float val = next_v;
        if (tid < dk) {
            key[tid] = next_k;
            if (OUT) query[tid] = next_q;
        }
        __syncthreads();
        if (t + 1 < stop) fetch(t + 1);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < R; i += 4) {
            const floatx4 k4 = *(const floatx4*)(key + row0 + i), q4 = *(const floatx4*)(query + row0 + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (row0 + i + e >= dk) continue;
                x[i + e] = fmaf(k4[e], val, reset ? 0.0f : g * x[i + e]);
                if (OUT) sum = fmaf(q4[e], x[i + e], sum);
            }
        }
        if (reset) cut = 1.0f; else factor *= g;
        if (OUT) part[tid] = sum;
        __syncthreads();
        if (OUT && tid < DVT && on) {
#pragma unroll
            for (int i = 1; i < RG; ++i) sum += part[tid + DVT * i];
            o[(int64_t)t * o_t + col] = (T)(scale * sum);
        }
        // (`part` is written again behind the next step's first barrier)
    }
#pragma unroll
    for (int i = 0; i < R; ++i) if (on && row0 + i < dk) state[(size_t)(row0 + i) * dv + col] = x[i];
    return make_float2(factor, cut);
}

// OUT: outputs and the state; else what every segment adds to the state.  VEC: 16-byte loads, a step's stride of less
// than 2^25 bytes (a chunk's offsets are 32 bits from a base that all threads share).
template <class T, int DK, int DVT, bool OUT, bool VEC>
__global__ __launch_bounds__(256, (DecayLds<T, DK, DVT, OUT>::RESIDENT)) void decay_chunk_kernel(DecayArgs p)
{
    typedef DecayMma<T> M;
    typedef typename M::Frag Frag;
    typedef DecayLds<T, DK, DVT, OUT> L;
    constexpr int C = M::C, FE = M::FE, KS = M::KS, KROW = L::KROW, CROW = L::CROW;
    constexpr int MT = DK / 16, NT = DVT / 64, IT = C / 16, JS = C / KS;     // state tiles a column; columns tiles a wavefront; step tiles; depth of a chunk
    constexpr int KB = (C / FE) * (DK / FE), VB = (C / FE) * (DVT / FE);     // FE x FE blocks of keys and values
    constexpr int BL = (KB + VB + 255) / 256, QL = C * (DK / FE) / 256;      // blocks and query vectors a thread
    extern __shared__ __attribute__((aligned(256))) char decay_lds[];
    char* const ldsq = decay_lds + L::Q; char* const ldsk = decay_lds + L::K; char* const ldskt = decay_lds + L::KT; char* const ldsvt = decay_lds + L::VT;
    float* const pw = (float*)(decay_lds + L::END);          // powers 0 .. C
    float* const wend = pw + C + 4;                          // weight of step j in the state behind the chunk
    uint64_t* const flags = (uint64_t*)(wend + C + 4);       // [0]: steps with a flag, [1]: a value is not finite, [2]: a score or query times state is not
    float* const reach = (float*)(flags + 4);                // OUT: scale times power i + 1: what step i sees of the state
    floatx4* const near = (floatx4*)(reach + C + 4);         // OUT: scale times the powers between a lane's steps of two tiles, see below

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ln = lane & 15, lg = lane >> 4;
    const int tiles = (p.dv + DVT - 1) / DVT;
    // neighbours (column tiles, heads of one key head) on one die: their keys and values meet in its cache
    const uint32_t total = gridDim.x, xcd = blockIdx.x & 7, per = total >> 3, more = total & 7;
    uint32_t id = xcd * per + (xcd < more ? xcd : more) + (blockIdx.x >> 3);
    const int tile = id % tiles; id /= tiles;
    const int grp = p.H / p.KV;
    const int hg = id % grp; id /= grp;
    const int seg = id % p.segments; id /= p.segments;
    const int hk = id % p.KV, b = id / p.KV, h = hk * grp + hg;
    const int bh = b * p.H + h, col0 = tile * DVT;
    const int len = decay_length(p, b);
    const int begin = seg * p.segment_steps, end = begin + min(p.segment_steps, len - begin);      // (not behind `begin`: none)
    const bool split = p.segments > 1;
    if (OUT && split && begin >= end) return;                // (the scan has the state)

    for (int n = tid; n <= C; n += 256) {
        double g = (double)p.decay[h], r = 1.0;
        for (int e = n; e; e >>= 1, g *= g) if (e & 1) r *= g;
        pw[n] = (float)r;
        if (OUT && n > 0) reach[n - 1] = p.scale * (float)r;
    }
    if constexpr (OUT) {
        // Lane: step ln of its tile, steps 4 lg .. of the other.  [0]: the same tile (zero above the diagonal); [1]: the
        // tile in front of it; further ones by another power of 16 steps a tile.
        __syncthreads();
        if (wave == 0)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int n = ln - 4 * lg - r;
                near[2 * lane][r] = n >= 0 ? p.scale * pw[n] : 0.0f;
                near[2 * lane + 1][r] = p.scale * pw[16 + n];
            }
    }
    // A thread's number that the compiler takes for a new one: addresses made from it are made where they are used (a few
    // instructions each); held across the loop, all of them together take more registers than there are.
    auto fresh = [](int x) { asm volatile("" : "+v"(x)); return x; };
    const size_t state = (size_t)p.dk * p.dv;
    floatx4 S[MT][NT];
    {
        const float* src = !OUT ? nullptr : split ? p.seg_state + ((size_t)bh * p.segments + seg) * state : p.s_in ? p.s_in + bh * state : nullptr;
        if (OUT && !split && p.done && len > 0 && p.done[b]) src = nullptr;       // the first step starts anew: what is there is not read
        const int me = fresh(lane);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = decay_row<T>(m, 4 * (me >> 4) + r), col = col0 + decay_row<T>(wave * NT + n, me & 15);
                    S[m][n][r] = src && row < p.dk && col < p.dv ? src[(size_t)row * p.dv + col] : 0.0f;
                }
    }
    const T* const q = (const T*)p.q + (int64_t)b * p.q_b + (int64_t)h * p.dk;
    const T* const k = (const T*)p.k + (int64_t)b * p.k_b + (int64_t)hk * p.dk;
    const T* const v = (const T*)p.v + (int64_t)b * p.v_b + (int64_t)hk * p.dv + col0;
    T* const o = (T*)p.out + (int64_t)b * p.o_b + (int64_t)h * p.dv + col0;
    const int dvt = min(DVT, p.dv - col0);

    // Block `at` of keys or values: FE steps from j on, FE elements from d on.  The order spreads a wavefront's writes of
    // both layouts over the banks and keeps 128 bytes of a row together in its reads.
    auto block_j = [](int at) { return ((at & 1) | ((at >> 4 & 3) << 1)) * FE; };
    auto block_d = [](int at) { return ((at >> 1 & 7) | (at >> 6 << 3)) * FE; };
    u32x4 blk[BL][FE], qv[OUT && !VEC ? QL : 1];
    uint8_t flag = 0;
    auto fetch = [&](int t0, int c) __attribute__((always_inline)) {                        // steps t0 .. t0 + c; behind them and behind the dimensions: any value of the array
        const int me = fresh(lane);
#pragma unroll
        for (int i = 0; i < BL; ++i) {
            const int first = wave * 64 + 256 * i, idx = first + me;
            const bool is_v = first >= KB;                   // (KB is whole wavefronts)
            const int at = is_v ? idx - KB : idx, j0 = block_j(at), d = block_d(at), dim = is_v ? dvt : p.dk;
            if (first >= KB + VB) continue;
            const int64_t step = is_v ? p.v_t : p.k_t;
            const T* const base = (is_v ? v : k) + (int64_t)t0 * step;
            if constexpr (VEC) {
                const uint32_t dd = min(d, dim - FE);
                if (c == C) {
                    const uint32_t one = (uint32_t)step * (uint32_t)sizeof(T);
                    uint32_t off = (uint32_t)(j0 * step + dd) * (uint32_t)sizeof(T);
#pragma unroll
                    for (int j = 0; j < FE; ++j, off += one) blk[i][j] = *(const u32x4*)((const char*)base + off);
                } else
#pragma unroll
                    for (int j = 0; j < FE; ++j) blk[i][j] = *(const u32x4*)((const char*)base + (uint32_t)(min(j0 + j, c - 1) * step + dd) * (uint32_t)sizeof(T));
            } else
#pragma unroll
                for (int j = 0; j < FE; ++j) blk[i][j] = decay_load16<T>(base + min(j0 + j, c - 1) * step, d, dim);
        }
        if constexpr (OUT && !VEC)
#pragma unroll
            for (int i = 0; i < QL; ++i) {
                const int idx = tid + 256 * i, j = min(idx / (DK / FE), c - 1), d = idx % (DK / FE) * FE;
                qv[i] = decay_load16<T>(q + (t0 + j) * p.q_t, d, p.dk);
            }
        flag = 0;
        if (p.done && tid < c) flag = p.done[(int64_t)(t0 + tid) * p.B + b];
    };
    // The queries go straight to LDS, 64 pieces of 16 bytes at a time: lane l's lands at place l, so it fetches the piece
    // that belongs there.  What stands behind the steps and behind key_dim is a repetition: outputs of steps that are not
    // there are not stored, and the keys are zero there.
    const uint32_t ldsq_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)ldsq;
    auto fetch_q = [&](int t0, int c) __attribute__((always_inline)) {
        if constexpr (OUT && VEC) {
            const T* const base = q + (int64_t)t0 * p.q_t;
            const int me = fresh(lane);
#pragma unroll
            for (int i = 0; i < C * KROW / 4096; ++i) {
                const int at = (wave * (C * KROW / 4096) + i) * 1024, byte = at + me * 16;
                int j, piece;
                if constexpr (KROW == 128) {
                    const int line = byte >> 8, y = (me & 15) ^ (line & 7);
                    j = 2 * line + (y >> 3); piece = y & 7;
                } else {
                    j = byte / KROW;
                    const int slot = byte / 16 % (KROW / 16);
                    piece = (slot & ~15) | ((slot ^ j) & 15);
                }
                g2lds16((const char*)base + (uint32_t)(min(j, c - 1) * p.q_t + min(piece * FE, p.dk - FE)) * (uint32_t)sizeof(T), ldsq_at + at);
            }
        }
    };
    auto stage = [&](int c) __attribute__((always_inline)) {
        uint32_t seen = 0;
        const u32x4 zero = {0, 0, 0, 0};
        const int me = fresh(lane);
#pragma unroll
        for (int i = 0; i < BL; ++i) {
            const int first = wave * 64 + 256 * i, idx = first + me;
            const bool is_v = first >= KB;
            const int at = is_v ? idx - KB : idx, j0 = block_j(at), d = block_d(at);
            if (first >= KB + VB) continue;
            if (c < C)
#pragma unroll
                for (int j = 0; j < FE; ++j) if (j0 + j >= c) blk[i][j] = zero;
            if (VEC && (is_v ? dvt < DVT : p.dk < DK)) {
                if (d >= (is_v ? dvt : p.dk))
#pragma unroll
                    for (int j = 0; j < FE; ++j) blk[i][j] = zero;
            }
#pragma unroll
            for (int j = 0; j < FE; ++j) {
                const u32x4 w = blk[i][j];
                seen = decay_magnitude<T>(decay_magnitude<T>(decay_magnitude<T>(decay_magnitude<T>(seen, w.x), w.y), w.z), w.w);
                if (OUT && !is_v) *(u32x4*)(ldsk + decay_at<KROW>(j0 + j, d / FE)) = w;
            }
            char* const to = is_v ? ldsvt : ldskt;
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    auto pick = [&](const u32x4& w) { return e == 0 ? w.x : e == 1 ? w.y : e == 2 ? w.z : w.w; };
                    *(u32x4*)(to + decay_at<CROW>(d + e, j0 / FE)) = u32x4{pick(blk[i][0]), pick(blk[i][1]), pick(blk[i][2]), pick(blk[i][3])};
                }
            } else {
                const int row = decay_place<T>(d);           // elements e: rows + (e & 3) + 16 (e >> 2)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    auto word = [&](const u32x4& w) { return e / 2 == 0 ? w.x : e / 2 == 1 ? w.y : e / 2 == 2 ? w.z : w.w; };
                    uint32_t o4[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j)              // the two steps' halves side by side
                        o4[j] = __builtin_amdgcn_perm(word(blk[i][2 * j + 1]), word(blk[i][2 * j]), e & 1 ? 0x07060302u : 0x05040100u);
                    *(u32x4*)(to + decay_at<CROW>(row + (e & 3) + 16 * (e >> 2), j0 / FE)) = u32x4{o4[0], o4[1], o4[2], o4[3]};
                }
            }
        }
        if constexpr (OUT && !VEC)
#pragma unroll
            for (int i = 0; i < QL; ++i) {
                const int idx = tid + 256 * i, j = idx / (DK / FE), d = idx % (DK / FE);
                *(u32x4*)(ldsq + decay_at<KROW>(j, d)) = qv[i];
            }
        if (wave == 0) {                                     // (c <= 64: one wavefront holds every step's flag)
            const uint64_t mask = __ballot(flag != 0);
            if (lane == 0) flags[0] = mask;
            if (lane < C) wend[lane] = lane < c && (mask >> lane >> 1) == 0 ? pw[c - 1 - lane] : 0.0f;
        }
        if (decay_not_finite<T>(seen)) flags[1] = 1;
    };
    auto uniform64 = [](uint64_t x) {
        return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
    };
    const uint32_t xk = decay_operand_x<KROW>(ln, lg), xc = decay_operand_x<CROW>(ln, lg);

    float factor = 1.0f, cut = 0.0f;                         // of the segment so far
    int t0 = begin, c = min(C, end - begin);
    if (c > 0) { fetch_q(t0, c); fetch(t0, c); }
    if (tid == 0) flags[1] = flags[2] = 0;
    __syncthreads();                                         // the table of powers
    while (c > 0) {
        stage(c);
        if constexpr (OUT && VEC) stage_wait();              // (the queries')
        __syncthreads();
        const uint64_t mask = uniform64(flags[0]);
        if (uniform64(flags[1])) break;
        const int next = t0 + c, nc = min(C, end - next);

        floatx4 acc[IT][NT];
        if constexpr (OUT) {
            // scores, transposed: lane: step i = 16 it + ln, four consecutive steps j
            constexpr int SC = IT == 4 ? 4 : 1;              // tiles a wavefront: row `it` = wave of four, or one of two x two
            floatx4 sc[SC];
            const int it = IT == 4 ? wave : wave >> 1;
#pragma unroll
            for (int x = 0; x < SC; ++x) sc[x] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int d = 0; d < DK / KS; ++d) {
                const Frag fq = *(const Frag*)(ldsq + decay_operand<KROW>(xk, 0, d) + it * 16 * KROW);
#pragma unroll
                for (int x = 0; x < SC; ++x) {
                    const int jt = IT == 4 ? x : wave & 1;   // (tiles above the diagonal too: the last wavefront needs all)
                    sc[x] = M::mma(*(const Frag*)(ldsk + decay_operand<KROW>(xk, 0, d) + jt * 16 * KROW), fq, sc[x]);
                }
            }
            __syncthreads();                                 // keys are read: scores take their place
            if (nc > 0) fetch(next, nc);                     // on its way while the rest is multiplied
            // NaN if a score, or below a query times the state, is not finite.  (Twice the score: the nearest bf16 of a finite
            // one may be infinite, too.)
            float none = 0.0f;
#pragma unroll
            for (int x = 0; x < SC; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) none = fmaf(sc[x][r] + sc[x][r], 0.0f, none);
            {
                const int i = 16 * it + ln;
                const floatx4 same = near[2 * lane], before = near[2 * lane + 1];
                const float p16 = pw[16];
                float far = 1.0f;                            // p16 ^ (it - jt - 1), from the nearest tile on
#pragma unroll
                for (int x = SC - 1; x >= 0; --x) {
                    const int jt = IT == 4 ? x : wave & 1;
                    if (jt > it) sc[x] = floatx4{0.f, 0.f, 0.f, 0.f};
                    else if (jt == it) sc[x] *= same;
                    else {
                        sc[x] *= before * far;
                        far *= p16;
                    }
                }
                if (mask) {                                  // steps from the last flag on
                    const uint64_t upto = mask & ((2ull << i) - 1);
                    const int low = upto ? 63 - __builtin_clzll(upto) : 0;
#pragma unroll
                    for (int x = 0; x < SC; ++x)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (16 * (IT == 4 ? x : wave & 1) + 4 * lg + r < low) sc[x][r] = 0.0f;
                }
#pragma unroll
                for (int x = 0; x < SC; ++x) {
                    const int jt = IT == 4 ? x : wave & 1;
                    const floatx4 f = sc[x];
                    if constexpr (sizeof(T) == 4) *(floatx4*)(ldsk + decay_at<CROW>(i, 4 * jt + lg)) = f;
                    else {
                        char* const to = ldsk + decay_at<CROW>(i, 2 * jt + (lg >> 1)) + 8 * (lg & 1);
                        const bf16x4 hi = to_bf16x4(f);
                        const floatx4 rest = f - to_floatx4(hi);
                        const bf16x4 mid = to_bf16x4(rest);
                        *(bf16x4*)to = hi;
                        *(bf16x4*)(to + C * CROW) = mid;
                        *(bf16x4*)(to + 2 * C * CROW) = to_bf16x4(rest - to_floatx4(mid));
                    }
                }
            }
            // queries x state, transposed: lane: four consecutive columns, step i = 16 it + ln
#pragma unroll
            for (int it2 = 0; it2 < IT; ++it2)
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[it2][n] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int d = 0; d < DK / KS; ++d) {
                Frag fq[IT];
                float x[NT][8];                              // what is left of the state
#pragma unroll
                for (int it2 = 0; it2 < IT; ++it2) fq[it2] = *(const Frag*)(ldsq + decay_operand<KROW>(xk, it2, d));
                if constexpr (sizeof(T) == 2)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[n][e] = S[2 * d + (e >> 2)][n][e & 3];
#pragma unroll
                for (int part = 0; part < L::PARTS; ++part) {
                    Frag fs[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        if constexpr (sizeof(T) == 4) fs[n] = S[d][n];
                        else fs[n] = part < 2 ? decay_split8(x[n]) : decay_round8(x[n]);
                    }
#pragma unroll
                    for (int it2 = 0; it2 < IT; ++it2)
#pragma unroll
                        for (int n = 0; n < NT; ++n) acc[it2][n] = M::mma(fs[n], fq[it2], acc[it2][n]);
                }
                __builtin_amdgcn_sched_barrier(0);           // (the state's parts are made where they are used)
            }
#pragma unroll
            for (int it2 = 0; it2 < IT; ++it2)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) none = fmaf(acc[it2][n][r], 0.0f, none);
            if (none != none) flags[2] = 1;
#pragma unroll
            for (int it2 = 0; it2 < IT; ++it2) {
                const int i = 16 * it2 + ln;
                const float w = reach[i];
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[it2][n] *= w;
            }
            if (mask)                                        // (a uniform branch: most chunks have no flag)
#pragma unroll
                for (int it2 = 0; it2 < IT; ++it2)
                    if (mask & ((2ull << (16 * it2 + ln)) - 1))
#pragma unroll
                        for (int n = 0; n < NT; ++n) acc[it2][n] = floatx4{0.f, 0.f, 0.f, 0.f};
            __syncthreads();                                 // the scores are there, and the queries are read
            if (uniform64(flags[2])) break;
            if (nc > 0) fetch_q(next, nc);
        } else if (nc > 0) fetch(next, nc);

        // the values of the wavefront's columns
        Frag vt[NT][JS];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int ks = 0; ks < JS; ++ks) vt[n][ks] = *(const Frag*)(ldsvt + decay_operand<CROW>(xc, n, ks) + wave * NT * 16 * CROW);

        if constexpr (OUT) {
#pragma unroll
            for (int ks = 0; ks < JS; ++ks)
#pragma unroll
                for (int part = 0; part < L::PARTS; ++part)
#pragma unroll
                    for (int it2 = 0; it2 < IT; ++it2) {
                        if (ks * KS > 16 * it2) continue;
                        const Frag f = *(const Frag*)(ldsk + decay_operand<CROW>(xc, it2, ks) + part * C * CROW);
#pragma unroll
                        for (int n = 0; n < NT; ++n) acc[it2][n] = M::mma(vt[n][ks], f, acc[it2][n]);
                    }
#pragma unroll
            for (int it2 = 0; it2 < IT; ++it2) {
                const int i = 16 * it2 + ln;
                if (i >= c) continue;
                T* const row = o + (int64_t)(t0 + i) * p.o_t;
                if constexpr (sizeof(T) == 2 && NT == 2) {   // two tiles are eight consecutive columns
                    const int col = 32 * wave + 8 * lg;
                    if (p.vec_o && col + 8 <= dvt) {
                        *(bf16x8*)(row + col) = to_bf16x8(acc[it2][0], acc[it2][1]);
                        continue;
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int col = decay_row<T>(wave * NT + n, 4 * lg);
                    const floatx4 f = acc[it2][n];
                    if (p.vec_o && col + 4 <= dvt) {
                        if constexpr (sizeof(T) == 4) *(floatx4*)(row + col) = f;
                        else *(bf16x4*)(row + col) = to_bf16x4(f);
                    } else
#pragma unroll
                        for (int r = 0; r < 4; ++r) if (col + r < dvt) row[col + r] = (T)f[r];
                }
            }
        }

        // the state behind the chunk
        if (mask) {
            cut = 1.0f;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) S[m][n] = floatx4{0.f, 0.f, 0.f, 0.f};
        } else {
            const float g = pw[c];
            factor *= g;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) S[m][n] *= g;
        }
#pragma unroll
        for (int ks = 0; ks < JS; ++ks) {
            Frag w[L::PARTS][NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const floatx4 wa = *(const floatx4*)(wend + ks * KS + FE * lg);
                if constexpr (sizeof(T) == 4) w[0][n] = vt[n][ks] * wa;
                else {
                    const floatx4 wb = *(const floatx4*)(wend + ks * KS + FE * lg + 4);
                    const u32x4 u = __builtin_bit_cast(u32x4, vt[n][ks]);
                    float x[8] = {bf16_lo_f32(u.x) * wa[0], bf16_hi_f32(u.x) * wa[1], bf16_lo_f32(u.y) * wa[2], bf16_hi_f32(u.y) * wa[3],
                                  bf16_lo_f32(u.z) * wb[0], bf16_hi_f32(u.z) * wb[1], bf16_lo_f32(u.w) * wb[2], bf16_hi_f32(u.w) * wb[3]};
                    w[0][n] = decay_split8(x);
                    w[1][n] = decay_split8(x);
                    w[2][n] = decay_round8(x);
                }
            }
#pragma unroll
            for (int m = 0; m < MT; m += 4) {                // (eight products in a row that do not wait for one another)
                Frag fk[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) fk[x] = *(const Frag*)(ldskt + decay_operand<CROW>(xc, m + x, ks));
#pragma unroll
                for (int y = 0; y < L::PARTS; ++y)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int n = 0; n < NT; ++n) S[m + x][n] = M::mma(fk[x], w[y][n], S[m + x][n]);
            }
        }
        __syncthreads();                                     // everything staged is read
        t0 = next;
        c = nc;
    }

    if (OUT && split && t0 >= end) return;
    float* const dst = OUT && !split ? p.s_out + bh * state : p.seg_state + ((size_t)bh * p.segments + seg) * state;
    const int me = fresh(lane);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = decay_row<T>(m, 4 * (me >> 4) + r), col = col0 + decay_row<T>(wave * NT + n, me & 15);
                if (row < p.dk && col < p.dv) dst[(size_t)row * p.dv + col] = S[m][n][r];
            }
    if (t0 < end) {
        const float2 f = decay_walk<T, DK, DVT, OUT>(decay_lds, q, k, v, o, dst + col0, p.done ? p.done + b : nullptr, p.decay[h], p.scale,
                                                     p.q_t, p.k_t, p.v_t, p.o_t, p.B, p.dk, p.dv, dvt, t0, end);
        factor *= f.x;
        if (f.y != 0.0f) cut = 1.0f;
    }
    if (!OUT && tile == 0 && tid == 0) p.seg_factor[(size_t)bh * p.segments + seg] = make_float2(factor, cut);
}

// The states in front of the segments, in place of what the segments add, and the state behind the last.
__global__ __launch_bounds__(256) void decay_scan_kernel(DecayArgs p)
{
    const size_t state = (size_t)p.dk * p.dv;
    const uint32_t blocks = (uint32_t)((state + 255) / 256);
    const uint32_t bh = blockIdx.x / blocks;
    const size_t at = (size_t)(blockIdx.x % blocks) * 256 + threadIdx.x;
    if (at >= state) return;
    // (where the first step starts anew what is there is not read: if it is no number, the first segment would be walked)
    const uint32_t b = bh / p.H;
    float s = p.s_in && !(p.done && decay_length(p, b) > 0 && p.done[b]) ? p.s_in[bh * state + at] : 0.0f;
    float* seg = p.seg_state + (size_t)bh * p.segments * state + at;
    const float2* f = p.seg_factor + (size_t)bh * p.segments;
    const bool forgets = p.decay[bh % p.H] == 0.0f;
    constexpr int U = 8;
    for (int i = 0; i < p.segments; i += U) {
        float add[U];
#pragma unroll
        for (int u = 0; u < U; ++u) if (i + u < p.segments) add[u] = seg[(i + u) * state];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u < p.segments) {
                seg[(i + u) * state] = s;
                const float2 g = f[i + u];
                // (a power too small for a number does not make an infinity NaN)
                s = (g.y != 0.0f ? 0.0f : __builtin_isinf(s) && !forgets ? copysignf(1.0f, g.x) * s : g.x * s) + add[u];
            }
    }
    p.s_out[bh * state + at] = s;
}

// ---- choice and layout of a call ----

struct DecayPlan {
    bool chunks;                 // else step by step
    int dk, dvt;                 // the kernel's sizes
    int segments, segment_steps;
    size_t factor_at, workspace; // bytes: where the factors stand, all
};

// Steps up to which the recurrence is walked: a step is a chain of two barriers, where a chunk costs the same for one step
// as for all of its own.  9 steps walked and as a chunk, us: 128 rows of 4 heads of 64 x 64 15.2 and 12.2 (fp32), 12.3 and
// 12.1 (bf16); 64 rows of 16 heads of 128 x 128 57.6 and 56.5 (fp32), 55.6 and 47.9 (bf16); 4 rows of them 12.6 and 14.5;
// 8 rows of 8 heads of 256 x 256 22.8 and 19.4 (bf16).  12 steps: a chunk everywhere.
constexpr int DECAY_SHORT = 8;

static inline DecayPlan decay_plan(int dtype, int T, int B, int H, int dk, int dv)
{
    DecayPlan q{};
    q.segments = 1; q.segment_steps = T;
    q.chunks = T > DECAY_SHORT;
    if (!q.chunks) return q;
    q.dk = dk <= 64 ? 64 : dk <= 128 ? 128 : 256;
    q.dvt = dv <= 64 || q.dk == 256 ? 64 : 128;
    const int C = dtype == SEED_DTYPE_FP32 ? DecayMma<float>::C : DecayMma<__bf16>::C;
    // Two workgroups a compute unit are wanted.  Fewer states than that: the time axis in segments, but of no less than
    // four chunks (a segment's keys and values are read once more, its state travels four times).
    const int64_t units = (int64_t)B * H * ((dv + q.dvt - 1) / q.dvt);
    const int64_t want = (512 + units - 1) / units, most = T / (4 * C);
    const int64_t n = want < most ? want : most;
    if (n > 1) {
        const int steps = (int)(((T + n - 1) / n + C - 1) / C * C);
        q.segments = (int)(((int64_t)T + steps - 1) / steps); q.segment_steps = steps;
    }
    if (q.segments > 1) {
        q.factor_at = ((size_t)B * H * q.segments * dk * dv * sizeof(float) + 255) / 256 * 256;
        q.workspace = q.factor_at + (size_t)B * H * q.segments * sizeof(float2);
    }
    return q;
}

template <class T, int DK, int DVT, bool VEC>
static hipError_t decay_launch_chunks(const DecayArgs& p, hipStream_t s)
{
    const unsigned tiles = (p.dv + DVT - 1) / DVT, grid = (unsigned)((size_t)p.B * p.H * p.segments * tiles);
    auto go = [&](auto out) -> hipError_t {
        constexpr bool OUT = decltype(out)::value;
        constexpr size_t lds = DecayLds<T, DK, DVT, OUT>::BYTES;
        const auto kernel = decay_chunk_kernel<T, DK, DVT, OUT, VEC>;
        static std::atomic<uint64_t> asked{0};
        const hipError_t e = op_allow_lds((const void*)kernel, lds, asked);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), lds, s, p);
        return hipSuccess;
    };
    if (p.segments > 1) {
        hipError_t e = go(std::false_type{});
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(decay_scan_kernel, dim3((unsigned)((size_t)p.B * p.H * (((size_t)p.dk * p.dv + 255) / 256))), dim3(256), 0, s, p);
    }
    return go(std::true_type{});
}

template <class T>
static hipError_t decay_launch(const DecayArgs& p, const DecayPlan& q, hipStream_t s)
{
    if (q.chunks && p.vec_in) {
        if (q.dk == 64) return q.dvt == 64 ? decay_launch_chunks<T, 64, 64, true>(p, s) : decay_launch_chunks<T, 64, 128, true>(p, s);
        if (q.dk == 128) return q.dvt == 64 ? decay_launch_chunks<T, 128, 64, true>(p, s) : decay_launch_chunks<T, 128, 128, true>(p, s);
        return decay_launch_chunks<T, 256, 64, true>(p, s);
    }
    if (q.chunks) {                                          // element by element: one width of columns is enough
        if (q.dk == 64) return decay_launch_chunks<T, 64, 64, false>(p, s);
        if (q.dk == 128) return decay_launch_chunks<T, 128, 64, false>(p, s);
        return decay_launch_chunks<T, 256, 64, false>(p, s);
    }
    const unsigned grid = (unsigned)((size_t)p.B * p.H * ((p.dv + DECAY_COLS - 1) / DECAY_COLS));
    if (p.dk <= 64) hipLaunchKernelGGL((decay_recurrent_kernel<T, 64>), dim3(grid), dim3(256), 0, s, p);
    else if (p.dk <= 128) hipLaunchKernelGGL((decay_recurrent_kernel<T, 128>), dim3(grid), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((decay_recurrent_kernel<T, 256>), dim3(grid), dim3(256), 0, s, p);
    return hipSuccess;
}

}  // namespace seedinf
