// The stand-alone operators' C entry points (include/seedinf.h): checks, workspaces, launches.
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>

#include "op_decay.h"
#include "op_norm.h"
#include "op_sample.h"

using namespace seedinf;

// Text of the calling thread's last failed operator call: a plain array, so that reporting an error cannot fail.
static thread_local char g_op_err[256] = "";

static seed_status_t op_fail(seed_status_t st, const char* format, ...)
{
    va_list args;
    va_start(args, format);
    vsnprintf(g_op_err, sizeof g_op_err, format, args);
    va_end(args);
    return st;
}

static seed_status_t op_launched()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SEED_OK : op_fail(SEED_ERR_DEVICE, "launch failed: %s", hipGetErrorString(e));
}

static bool op_overlap(const void* a, size_t na, const void* b, size_t nb)
{
    const char* pa = (const char*)a;
    const char* pb = (const char*)b;
    return a && b && na && nb && pa < pb + nb && pb < pa + na;
}

// n places `stride` elements apart: do they end within 2^46 elements, so that no sum of two such extents leaves 64 bits?
static bool op_reaches(int64_t n, int64_t stride) { return stride >= 0 && (n <= 1 || stride <= ((int64_t)1 << 46) / (n - 1)); }

static bool op_aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

static seed_status_t op_check_workspace(size_t need, const void* workspace, size_t have)
{
    if (!need) return SEED_OK;
    if (!workspace || have < need) return op_fail(SEED_ERR_INVALID_ARG, "the call needs %zu bytes of workspace, %zu are given", need, workspace ? have : 0);
    if (!op_aligned(workspace, 256)) return op_fail(SEED_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    return SEED_OK;
}

static bool op_dtype_ok(int32_t dtype) { return dtype == SEED_DTYPE_FP32 || dtype == SEED_DTYPE_BF16; }

extern "C" const char* seed_op_last_error(void) { return g_op_err; }

// ---- linear attention with decay ----

static seed_status_t decay_check(const seed_decay_t* d)
{
    if (!d) return op_fail(SEED_ERR_INVALID_ARG, "desc is NULL");
    if (d->struct_size != sizeof(seed_decay_t)) return op_fail(SEED_ERR_INVALID_ARG, "desc->struct_size is not sizeof(seed_decay_t)");
    if (!op_dtype_ok(d->dtype)) return op_fail(SEED_ERR_INVALID_ARG, "dtype must be SEED_DTYPE_FP32 or SEED_DTYPE_BF16");
    if (d->steps < 0 || d->rows < 0) return op_fail(SEED_ERR_INVALID_ARG, "steps or rows is negative");
    if (d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads) return op_fail(SEED_ERR_INVALID_ARG, "kv_heads must divide heads, both positive");
    if (d->key_dim < 1 || d->key_dim > 256 || d->value_dim < 1 || d->value_dim > 256)
        return op_fail(SEED_ERR_INVALID_ARG, "key_dim and value_dim must be 1 .. 256");
    const int64_t strides[][2] = {{d->q_step, d->q_row}, {d->k_step, d->k_row}, {d->v_step, d->v_row}, {d->out_step, d->out_row}};
    for (const auto& s : strides)
        if (s[0] > ((int64_t)1 << 44) || s[1] > ((int64_t)1 << 44) || !op_reaches(d->steps, s[0]) || !op_reaches(d->rows, s[1]))
            return op_fail(SEED_ERR_INVALID_ARG, "a stride is negative or too large");
    // a launch's threads stay below 2^32
    if ((int64_t)d->rows * d->heads > ((int64_t)1 << 21)) return op_fail(SEED_ERR_INVALID_ARG, "rows * heads is more than 2^21");
    return SEED_OK;
}

// [steps, rows, width] elements with strides: do two of them share memory?  Two with the same strides that lie beside
// each other (parts of one projection's output) do not; any other overlap of their extents counts as one.
struct StridedArray { const void* p; int64_t step, row, width; };
static bool strided_overlap(const StridedArray& a, const StridedArray& b, int64_t T, int64_t B, size_t size)
{
    auto extent = [&](const StridedArray& x) { return (size_t)((T - 1) * x.step + (B - 1) * x.row + x.width) * size; };
    if (!op_overlap(a.p, extent(a), b.p, extent(b))) return false;
    const int64_t bytes = (const char*)b.p - (const char*)a.p, w = a.width > b.width ? a.width : b.width;
    if (a.step != b.step || a.row != b.row || bytes % (int64_t)size) return true;
    // the outer stride steps over whole runs of the inner one, the inner one over whole rows
    const bool rows_outer = B > 1 && (T == 1 || a.row > a.step);
    const int64_t so = rows_outer ? a.row : a.step, no = rows_outer ? B : T, si = rows_outer ? a.step : a.row, ni = rows_outer ? T : B;
    if ((ni > 1 && si < w) || (no > 1 && so < (ni - 1) * si + w)) return true;
    auto floor_div = [](int64_t x, int64_t y) { return x / y - (x % y < 0); };
    const int64_t delta = bytes / (int64_t)size;
    const int64_t o0 = no > 1 ? floor_div(delta, so) : 0;
    for (int64_t o = o0; o <= o0 + (no > 1); ++o) {                 // b starts between two of a's outer places ...
        if (o >= no || o <= -no) continue;
        const int64_t rest = delta - o * so, i0 = ni > 1 ? floor_div(rest, si) : 0;
        for (int64_t i = i0; i <= i0 + (ni > 1); ++i)               // ... and between two of the inner ones
            if (i < ni && i > -ni && rest - i * si < a.width && rest - i * si > -b.width) return true;
    }
    return false;
}

extern "C" size_t seed_op_decay_workspace(const seed_decay_t* desc)
{
    if (decay_check(desc) != SEED_OK || desc->rows == 0) return 0;
    return decay_plan(desc->dtype, desc->steps, desc->rows, desc->heads, desc->key_dim, desc->value_dim).workspace;
}

extern "C" seed_status_t seed_op_decay(const seed_decay_t* d, const void* q, const void* k, const void* v, const float* decay,
                                       const uint8_t* done, const int32_t* lengths, const float* state_in, void* out,
                                       float* state_out, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    seed_status_t st = decay_check(d);
    if (st != SEED_OK) return st;
    if (d->rows == 0) return SEED_OK;
    if (!decay || !state_out || (d->steps > 0 && (!q || !k || !v || !out)))
        return op_fail(SEED_ERR_INVALID_ARG, "q, k, v, decay, out and state_out are required");
    const size_t size = op_dtype_size(d->dtype);
    if (!op_aligned(q, size) || !op_aligned(k, size) || !op_aligned(v, size) || !op_aligned(out, size) || !op_aligned(state_in, 4) || !op_aligned(state_out, 4) ||
        !op_aligned(decay, 4) || !op_aligned(lengths, 4))
        return op_fail(SEED_ERR_INVALID_ARG, "an array is not aligned to its element");
    const size_t state_bytes = (size_t)d->rows * d->heads * d->key_dim * d->value_dim * sizeof(float);
    if (state_in != state_out && op_overlap(state_in, state_bytes, state_out, state_bytes))
        return op_fail(SEED_ERR_ALIASING, "state_out overlaps state_in without being it");
    const struct { const void* p; size_t bytes; } small[] = {{decay, (size_t)d->heads * 4}, {done, (size_t)d->steps * d->rows}, {lengths, (size_t)d->rows * 4}};
    for (const auto& a : small)
        if (op_overlap(a.p, a.bytes, state_out, state_bytes)) return op_fail(SEED_ERR_ALIASING, "state_out overlaps decay, done or lengths");
    const size_t need = seed_op_decay_workspace(d);
    if (need && (op_overlap(workspace, need, state_in, state_bytes) || op_overlap(workspace, need, state_out, state_bytes)))
        return op_fail(SEED_ERR_ALIASING, "the workspace overlaps a state");
    for (const auto& a : small)
        if (op_overlap(a.p, a.bytes, workspace, need)) return op_fail(SEED_ERR_ALIASING, "the workspace overlaps decay, done or lengths");
    if (d->steps > 0) {
        const StridedArray arrays[] = {{out, d->out_step, d->out_row, (int64_t)d->heads * d->value_dim},
                                       {q, d->q_step, d->q_row, (int64_t)d->heads * d->key_dim},
                                       {k, d->k_step, d->k_row, (int64_t)d->kv_heads * d->key_dim},
                                       {v, d->v_step, d->v_row, (int64_t)d->kv_heads * d->value_dim}};
        for (const StridedArray& a : arrays) {
            if (a.p != out && strided_overlap(arrays[0], a, d->steps, d->rows, size)) return op_fail(SEED_ERR_ALIASING, "out overlaps q, k or v");
            const size_t extent = (size_t)((d->steps - 1) * a.step + (d->rows - 1) * a.row + a.width) * size;
            if (op_overlap(a.p, extent, state_out, state_bytes)) return op_fail(SEED_ERR_ALIASING, "state_out overlaps q, k, v or out");
            if (need && op_overlap(a.p, extent, workspace, need)) return op_fail(SEED_ERR_ALIASING, "the workspace overlaps q, k, v or out");
            if (a.p != out) continue;
            if (op_overlap(out, extent, state_in, state_bytes)) return op_fail(SEED_ERR_ALIASING, "out overlaps state_in");
            for (const auto& b : small)
                if (op_overlap(out, extent, b.p, b.bytes)) return op_fail(SEED_ERR_ALIASING, "out overlaps decay, done or lengths");
        }
        if (out == q || out == k || out == v) return op_fail(SEED_ERR_ALIASING, "out overlaps q, k or v");
        // out's rows lie apart: one of its strides steps over a whole row, the other over all rows of the first
        const bool rows_outer = d->steps == 1 || (d->rows > 1 && d->out_row > d->out_step);
        const int64_t w = arrays[0].width, so = rows_outer ? d->out_row : d->out_step, no = rows_outer ? d->rows : d->steps;
        const int64_t si = rows_outer ? d->out_step : d->out_row, ni = rows_outer ? d->steps : d->rows;
        if ((ni > 1 && si < w) || (no > 1 && so < (ni - 1) * si + w)) return op_fail(SEED_ERR_ALIASING, "out's strides make its rows overlap");
    }
    if ((st = op_check_workspace(need, workspace, workspace_bytes)) != SEED_OK) return st;
    DecayArgs p{};
    p.q = q; p.k = k; p.v = v; p.decay = decay; p.done = done; p.lengths = lengths; p.s_in = state_in; p.out = out; p.s_out = state_out;
    p.q_t = d->q_step; p.q_b = d->q_row; p.k_t = d->k_step; p.k_b = d->k_row; p.v_t = d->v_step; p.v_b = d->v_row; p.o_t = d->out_step; p.o_b = d->out_row;
    p.T = d->steps; p.B = d->rows; p.H = d->heads; p.KV = d->kv_heads; p.dk = d->key_dim; p.dv = d->value_dim; p.scale = d->scale;
    p.vec_state = d->value_dim % 4 == 0 && op_aligned(state_in, 16) && op_aligned(state_out, 16);
    const DecayPlan plan = decay_plan(d->dtype, d->steps, d->rows, d->heads, d->key_dim, d->value_dim);
    p.segments = plan.segments; p.segment_steps = plan.segment_steps;
    if (plan.workspace) {
        p.seg_state = (float*)workspace;
        p.seg_factor = (float2*)((char*)workspace + plan.factor_at);
    }
    // n elements from every head on, at a time
    auto whole = [&](const void* a, int64_t step, int64_t row, int dim, int n) {
        return op_aligned(a, n * size) && dim % n == 0 && (d->steps == 1 || step % n == 0) && (d->rows == 1 || row % n == 0);
    };
    const int n16 = (int)(16 / size);
    const int64_t near = ((int64_t)1 << 25) / (int64_t)size;
    p.vec_in = whole(q, p.q_t, p.q_b, p.dk, n16) && whole(k, p.k_t, p.k_b, p.dk, n16) && whole(v, p.v_t, p.v_b, p.dv, n16) && p.q_t < near && p.k_t < near && p.v_t < near;
    p.vec_o = whole(out, p.o_t, p.o_b, p.dv, n16);
    const hipError_t e = d->dtype == SEED_DTYPE_FP32 ? decay_launch<float>(p, plan, (hipStream_t)hip_stream) : decay_launch<__bf16>(p, plan, (hipStream_t)hip_stream);
    if (e != hipSuccess) return op_fail(SEED_ERR_DEVICE, "launch failed: %s", hipGetErrorString(e));
    return op_launched();
}

// ---- group normalisation ----

static seed_status_t norm_check(int32_t dtype, int32_t rows, int32_t points, int32_t channels, int32_t groups)
{
    if (!op_dtype_ok(dtype)) return op_fail(SEED_ERR_INVALID_ARG, "dtype must be SEED_DTYPE_FP32 or SEED_DTYPE_BF16");
    if (rows < 0 || points < 0) return op_fail(SEED_ERR_INVALID_ARG, "rows or points is negative");
    if (channels < 1 || groups < 1 || channels % groups) return op_fail(SEED_ERR_INVALID_ARG, "groups must divide channels, both positive");
    if ((int64_t)points * channels >= (int64_t)1 << 31) return op_fail(SEED_ERR_INVALID_ARG, "points * channels is 2^31 or more");
    if ((int64_t)rows * groups > (int64_t)1 << 23) return op_fail(SEED_ERR_INVALID_ARG, "rows * groups is more than 2^23");
    return SEED_OK;
}

extern "C" size_t seed_op_group_norm_workspace(int32_t dtype, int32_t rows, int32_t points, int32_t channels, int32_t groups)
{
    if (norm_check(dtype, rows, points, channels, groups) != SEED_OK || rows == 0 || points == 0) return 0;
    // whatever the arrays' alignment turns out to be
    size_t most = 0;
    const int size = (int)op_dtype_size(dtype);
    for (int vec = 16 / size; vec >= 1; vec /= 2) {
        const size_t n = norm_plan(rows, points, channels, groups, size, vec).workspace;
        if (n > most) most = n;
    }
    return most;
}

extern "C" seed_status_t seed_op_group_norm(int32_t dtype, int32_t rows, int32_t points, int32_t channels, int32_t groups, const void* x,
                                            const float* weight, const float* bias, float eps, int32_t activation, void* out,
                                            void* workspace, size_t workspace_bytes, void* hip_stream)
{
    seed_status_t st = norm_check(dtype, rows, points, channels, groups);
    if (st != SEED_OK) return st;
    if (!(eps >= 0.0f)) return op_fail(SEED_ERR_INVALID_ARG, "eps is negative");
    if (activation != SEED_ACT_NONE && activation != SEED_ACT_RELU && activation != SEED_ACT_SILU)
        return op_fail(SEED_ERR_INVALID_ARG, "activation must be SEED_ACT_NONE, SEED_ACT_RELU or SEED_ACT_SILU");
    if (rows == 0 || points == 0) return SEED_OK;
    if (!x || !out) return op_fail(SEED_ERR_INVALID_ARG, "x and out are required");
    const size_t size = op_dtype_size(dtype), bytes = (size_t)rows * points * channels * size;
    if (!op_aligned(x, size) || !op_aligned(out, size) || !op_aligned(weight, 4) || !op_aligned(bias, 4))
        return op_fail(SEED_ERR_INVALID_ARG, "an array is not aligned to its element");
    if ((x != out && op_overlap(x, bytes, out, bytes)) || op_overlap(weight, (size_t)channels * 4, out, bytes) || op_overlap(bias, (size_t)channels * 4, out, bytes))
        return op_fail(SEED_ERR_ALIASING, "out overlaps x without being it, or weight or bias");
    const size_t need = seed_op_group_norm_workspace(dtype, rows, points, channels, groups), params = (size_t)channels * 4;
    if (need && (op_overlap(workspace, need, x, bytes) || op_overlap(workspace, need, out, bytes) || op_overlap(workspace, need, weight, params) || op_overlap(workspace, need, bias, params)))
        return op_fail(SEED_ERR_ALIASING, "the workspace overlaps an array");
    if ((st = op_check_workspace(need, workspace, workspace_bytes)) != SEED_OK) return st;
    int vec = (int)(16 / size);
    while (!op_aligned(x, vec * size) || !op_aligned(out, vec * size)) vec /= 2;
    const NormPlan plan = norm_plan(rows, points, channels, groups, (int)size, vec);
    NormArgs p{x, out, weight, bias, rows, points, channels, groups, eps, activation, op_aligned(weight, 16) && op_aligned(bias, 16)};
    if (dtype == SEED_DTYPE_FP32) norm_launch<float>(p, plan, workspace, (hipStream_t)hip_stream);
    else norm_launch<__bf16>(p, plan, workspace, (hipStream_t)hip_stream);
    return op_launched();
}

// ---- sampling ----

static seed_status_t sample_check(int32_t dtype, int32_t rows, int32_t choices)
{
    if (!op_dtype_ok(dtype)) return op_fail(SEED_ERR_INVALID_ARG, "dtype must be SEED_DTYPE_FP32 or SEED_DTYPE_BF16");
    if (rows < 0 || rows > 1 << 21) return op_fail(SEED_ERR_INVALID_ARG, "rows must be 0 .. 2^21");
    if (choices < 1 || choices > SEED_SAMPLE_MAX_CHOICES) return op_fail(SEED_ERR_INVALID_ARG, "choices must be 1 .. %d", SEED_SAMPLE_MAX_CHOICES);
    return SEED_OK;
}

extern "C" size_t seed_op_sample_workspace(int32_t dtype, int32_t rows, int32_t choices)
{
    if (sample_check(dtype, rows, choices) != SEED_OK) return 0;
    return 0;
}

// Everything that seed_op_sample refuses.
seed_status_t seedinf::op_sample_check(int32_t dtype, int32_t rows, int32_t choices, int64_t row_stride, const void* logits,
                                        const float* uniforms, const float* temperature, const int32_t* top_k, const float* top_p,
                                        const float* min_p, int32_t* token_out, float* logprob_out)
{
    seed_status_t st = sample_check(dtype, rows, choices);
    if (st != SEED_OK) return st;
    if (row_stride > (int64_t)1 << 44 || !op_reaches(rows, row_stride)) return op_fail(SEED_ERR_INVALID_ARG, "row_stride is negative or too large");
    if (rows == 0) return SEED_OK;
    if (!logits || !uniforms || !token_out) return op_fail(SEED_ERR_INVALID_ARG, "logits, uniforms and token_out are required");
    const size_t size = op_dtype_size(dtype), bytes = ((size_t)(rows - 1) * row_stride + choices) * size, row4 = (size_t)rows * 4;
    if (!op_aligned(logits, size)) return op_fail(SEED_ERR_INVALID_ARG, "logits is not aligned to its element");
    const void* in[] = {uniforms, temperature, top_k, top_p, min_p};
    for (const void* a : in) {
        if (!op_aligned(a, 4)) return op_fail(SEED_ERR_INVALID_ARG, "an array is not aligned to its element");
        if (op_overlap(a, row4, token_out, row4) || op_overlap(a, row4, logprob_out, row4)) return op_fail(SEED_ERR_ALIASING, "an output overlaps an input");
    }
    if (!op_aligned(token_out, 4) || !op_aligned(logprob_out, 4)) return op_fail(SEED_ERR_INVALID_ARG, "an array is not aligned to its element");
    if (op_overlap(logits, bytes, token_out, row4) || op_overlap(logits, bytes, logprob_out, row4) || op_overlap(token_out, row4, logprob_out, row4))
        return op_fail(SEED_ERR_ALIASING, "an output overlaps an input or the other output");
    return SEED_OK;
}

extern "C" seed_status_t seed_op_sample(int32_t dtype, int32_t rows, int32_t choices, int64_t row_stride, const void* logits,
                                        const float* uniforms, const float* temperature, const int32_t* top_k, const float* top_p,
                                        const float* min_p, int32_t* token_out, float* logprob_out, void* workspace,
                                        size_t workspace_bytes, void* hip_stream)
{
    seed_status_t st = op_sample_check(dtype, rows, choices, row_stride, logits, uniforms, temperature, top_k, top_p, min_p, token_out, logprob_out);
    if (st != SEED_OK || rows == 0) return st;
    if ((st = op_check_workspace(seed_op_sample_workspace(dtype, rows, choices), workspace, workspace_bytes)) != SEED_OK) return st;
    SampleArgs p{logits, row_stride, uniforms, temperature, top_k, top_p, min_p, token_out, logprob_out, rows, choices};
    const hipError_t e = dtype == SEED_DTYPE_FP32 ? sample_launch<float>(p, (hipStream_t)hip_stream) : sample_launch<__bf16>(p, (hipStream_t)hip_stream);
    if (e != hipSuccess) return op_fail(SEED_ERR_DEVICE, "launch failed: %s", hipGetErrorString(e));
    return op_launched();
}
