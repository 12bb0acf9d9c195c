// Rows of real values to 8-bit codes with one scale per row: gated activations and weight matrices (f8_quantize_rows), and the step
// between two blocks -- norm, gate and scale of a block's output, residual sum, norm of the next block (f8_norm_quantize).
//
//     t = r + beta * g(gate) * post(x);   v = pre(t)           or    v = act(x) * u
//     a = max |v|;  s = a / 127;  i = 127 / a;  q = floor(v * i + 1/2)
//
// Bound by memory traffic: every element is read and written once, and all a row needs besides is a few sums over it.
//
// The row kernels here take any width, alignment and row distance: one block per row, the passes over it (one per sum, then
// one that writes) read the row again, which then comes from the caches.
#include <math.h>

#include "f8_real.cuh"

namespace {

constexpr int ROW_THREADS = 256;

struct RowsParams {
    int c, act;
    long long ldx, ldu, ldy, ldq;
    const void *x, *u;
    int8_t *q;
    float *scale;
    void *y;
};

template <int ACT>
__device__ __forceinline__ float activate(float v) {
    if (ACT == F8_ACT_SILU) return v / (1.f + expf(-v));
    if (ACT == F8_ACT_GELU) return v * normcdff(v);      // relative precision for negative v too, which 1 + erf loses
    if (ACT == F8_ACT_SIGMOID) return 1.f / (1.f + expf(-v));
    if (ACT == F8_ACT_TANH) return tanhf(v);
    return v;
}

template <typename T, int ACT>
__global__ void __launch_bounds__(ROW_THREADS) quantize_rows_kernel(RowsParams p) {
    wait_for_stream();
    let_stream_go_on();
    __shared__ uint32_t room[32];
    const long long row = blockIdx.x;
    const T *x = (const T *)p.x + row * p.ldx, *u = p.u ? (const T *)p.u + row * p.ldu : nullptr;
    T *y = p.y ? (T *)p.y + row * p.ldy : nullptr;
    int8_t *q = p.q ? p.q + row * p.ldq : nullptr;
    auto value = [&](int i) {
        const float v = activate<ACT>(to_float(x[i]));
        return u ? v * to_float(u[i]) : v;
    };
    if (!q) {
        for (int i = threadIdx.x; i < p.c; i += ROW_THREADS) y[i] = from_float<T>(value(i));
        return;
    }
    uint32_t peak = 0;
    for (int i = threadIdx.x; i < p.c; i += ROW_THREADS) peak = max(peak, magnitude(value(i)));
    const RowScale s(block_reduce<ROW_THREADS>(peak, UMaxOp(), room));
    if (threadIdx.x == 0) p.scale[row] = s.scale;
    for (int i = threadIdx.x; i < p.c; i += ROW_THREADS) {
        const int code = s.code(value(i));
        q[i] = (int8_t)code;
        if (y) y[i] = from_float<T>((float)code * s.scale);
    }
}

struct NormParams {
    int c, post_norm, pre_norm, gate_act;
    float eps, weight_offset, branch_scale;
    long long ldx, ldg, ldr, lds, ldy, ldq;
    const void *x, *gate, *res, *post_w, *post_b, *pre_w, *pre_b;
    void *sum;
    int8_t *q;
    float *scale;
    void *y;
};

__device__ __forceinline__ float gate_value(float g, int act) {
    return act == F8_ACT_SIGMOID ? activate<F8_ACT_SIGMOID>(g) : act == F8_ACT_TANH ? activate<F8_ACT_TANH>(g) : g;
}

// z -> (z - mean) * rstd * (w + offset) + b
template <typename W>
struct Norm {
    const W *w, *b;
    float mean, rstd, offset;
    bool on;
    __device__ __forceinline__ float operator()(float z, int i) const {
        if (!on) return z;
        z = (z - mean) * rstd;
        if (w) z *= to_float(w[i]) + offset;
        if (b) z += to_float(b[i]);
        return z;
    }
};

template <typename T, typename W>
__global__ void __launch_bounds__(ROW_THREADS) norm_quantize_kernel(NormParams p) {
    wait_for_stream();
    let_stream_go_on();
    __shared__ float room[32];
    __shared__ uint32_t uroom[32];
    const long long row = blockIdx.x;
    const T *x = (const T *)p.x + row * p.ldx, *g = p.gate ? (const T *)p.gate + row * p.ldg : nullptr;
    const T *r = p.res ? (const T *)p.res + row * p.ldr : nullptr;
    T *sum = p.sum ? (T *)p.sum + row * p.lds : nullptr, *y = p.y ? (T *)p.y + row * p.ldy : nullptr;
    int8_t *q = p.q ? p.q + row * p.ldq : nullptr;
    // mean and 1 / deviation of what `f` gives over the row (the deviation from the mean: a second pass)
    auto measure = [&](int kind, auto f, float &mean, float &rstd) {
        mean = 0.f;
        rstd = 1.f;
        if (kind == F8_NORM_NONE) return;
        if (kind == F8_NORM_LAYER) {
            float s = 0.f;
            for (int i = threadIdx.x; i < p.c; i += ROW_THREADS) s += f(i);
            mean = block_reduce<ROW_THREADS>(s, SumOp(), room) / (float)p.c;
        }
        float s = 0.f;
        for (int i = threadIdx.x; i < p.c; i += ROW_THREADS) {
            const float z = f(i) - mean;
            s += z * z;
        }
        rstd = 1.f / sqrtf(block_reduce<ROW_THREADS>(s, SumOp(), room) / (float)p.c + p.eps);
    };
    Norm<W> post = {(const W *)p.post_w, (const W *)p.post_b, 0.f, 1.f, p.weight_offset, p.post_norm != F8_NORM_NONE};
    Norm<W> pre = {(const W *)p.pre_w, (const W *)p.pre_b, 0.f, 1.f, p.weight_offset, p.pre_norm != F8_NORM_NONE};
    measure(p.post_norm, [&](int i) { return to_float(x[i]); }, post.mean, post.rstd);
    auto total = [&](int i) {
        float z = post(to_float(x[i]), i);
        if (g) z *= gate_value(to_float(g[i]), p.gate_act);
        return fmaf(p.branch_scale, z, r ? to_float(r[i]) : 0.f);
    };
    measure(p.pre_norm, total, pre.mean, pre.rstd);
    RowScale s(0);
    if (q) {
        uint32_t peak = 0;
        for (int i = threadIdx.x; i < p.c; i += ROW_THREADS) peak = max(peak, magnitude(pre(total(i), i)));
        s = RowScale(block_reduce<ROW_THREADS>(peak, UMaxOp(), uroom));
        if (threadIdx.x == 0) p.scale[row] = s.scale;
    }
    for (int i = threadIdx.x; i < p.c; i += ROW_THREADS) {
        const float t = total(i), v = pre(t, i);
        if (sum) sum[i] = from_float<T>(t);
        if (q) {
            const int code = s.code(v);
            q[i] = (int8_t)code;
            if (y) y[i] = from_float<T>((float)code * s.scale);
        } else if (y) {
            y[i] = from_float<T>(v);
        }
    }
}

template <typename T>
cudaError_t launch_rows(const RowsParams &p, long long n, cudaStream_t st) {
    const dim3 grid((unsigned)n);
    switch (p.act) {
        case F8_ACT_SILU: return launch_early(quantize_rows_kernel<T, F8_ACT_SILU>, grid, ROW_THREADS, 0, st, p);
        case F8_ACT_GELU: return launch_early(quantize_rows_kernel<T, F8_ACT_GELU>, grid, ROW_THREADS, 0, st, p);
        default: return launch_early(quantize_rows_kernel<T, F8_ACT_NONE>, grid, ROW_THREADS, 0, st, p);
    }
}

template <typename T>
cudaError_t launch_norm(const NormParams &p, long long n, bool w32, cudaStream_t st) {
    const dim3 grid((unsigned)n);
    if (w32) return launch_early(norm_quantize_kernel<T, float>, grid, ROW_THREADS, 0, st, p);
    return launch_early(norm_quantize_kernel<T, T>, grid, ROW_THREADS, 0, st, p);
}

// Row distance: 0 stands for dense rows; false where rows would overlap or the matrix would pass what a pointer reaches.
bool row_distance(long long *ld, int c, long long n) {
    if (*ld == 0) *ld = c;
    return *ld >= c && *ld <= (1ll << 40) && (n <= 1 || *ld <= (1ll << 50) / n);
}

bool misaligned(const void *p, int size) { return ((uintptr_t)p & (uintptr_t)(size - 1)) != 0; }

}   // namespace

extern "C" {

f8_status f8_quantize_rows(const f8_rows_desc *desc, const void *x, const void *u, int8_t *q, float *scale, void *y, void *cuda_stream) {
    if (!desc) return f8_set_error(F8_ERR_NULL, "descriptor is NULL");
    f8_rows_desc d = *desc;
    if (d.n < 0 || d.n > 0x7fffffffll || d.c <= 0) return f8_set_error(F8_ERR_SHAPE, "n in 0 .. 2^31 - 1 and c > 0 are needed");
    const int size = real_size(d.dtype);
    if (!size) return f8_set_error(F8_ERR_DTYPE, "dtype must be F8_F32, F8_F16 or F8_BF16");
    if (d.act != F8_ACT_NONE && d.act != F8_ACT_SILU && d.act != F8_ACT_GELU)
        return f8_set_error(F8_ERR_UNSUPPORTED, "act must be F8_ACT_NONE, F8_ACT_SILU or F8_ACT_GELU");
    if (!row_distance(&d.ldx, d.c, d.n) || !row_distance(&d.ldu, d.c, d.n) || !row_distance(&d.ldy, d.c, d.n) || !row_distance(&d.ldq, d.c, d.n))
        return f8_set_error(F8_ERR_SHAPE, "a row distance is smaller than the row, or too large");
    if (d.n == 0) return F8_OK;
    if (!x || (!q && !y) || (q && !scale) || (!q && scale)) return f8_set_error(F8_ERR_NULL, "x, and q with scale or y, must not be NULL");
    if (misaligned(x, size) || misaligned(u, size) || misaligned(y, size) || misaligned(scale, 4))
        return f8_set_error(F8_ERR_ALIGN, "a pointer is not aligned to its element");
    if (f8_pending_timeout() != F8_OK) return F8_ERR_TIMEOUT;
    RowsParams p = {d.c, d.act, d.ldx, d.ldu, d.ldy, d.ldq, x, u, q, scale, y};
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = d.dtype == F8_F32 ? launch_rows<float>(p, d.n, st) : d.dtype == F8_F16 ? launch_rows<__half>(p, d.n, st) : launch_rows<__nv_bfloat16>(p, d.n, st);
    if (e != cudaSuccess) return f8_set_error(F8_ERR_CUDA, cudaGetErrorString(e));
    return F8_OK;
}

f8_status f8_norm_quantize(const f8_norm_desc *desc, const void *x, const void *gate, const void *residual, const void *post_w,
                           const void *post_b, const void *pre_w, const void *pre_b, void *residual_out, int8_t *q, float *scale,
                           void *y, void *cuda_stream) {
    if (!desc) return f8_set_error(F8_ERR_NULL, "descriptor is NULL");
    f8_norm_desc d = *desc;
    if (d.n < 0 || d.n > 0x7fffffffll || d.c <= 0) return f8_set_error(F8_ERR_SHAPE, "n in 0 .. 2^31 - 1 and c > 0 are needed");
    const int size = real_size(d.dtype);
    if (!size) return f8_set_error(F8_ERR_DTYPE, "dtype must be F8_F32, F8_F16 or F8_BF16");
    if (d.w_dtype != F8_F32 && d.w_dtype != d.dtype) return f8_set_error(F8_ERR_DTYPE, "w_dtype must be F8_F32 or dtype");
    if (d.post_norm < F8_NORM_NONE || d.post_norm > F8_NORM_LAYER || d.pre_norm < F8_NORM_NONE || d.pre_norm > F8_NORM_LAYER)
        return f8_set_error(F8_ERR_UNSUPPORTED, "a norm must be F8_NORM_NONE, F8_NORM_RMS or F8_NORM_LAYER");
    if (d.gate_act != F8_ACT_NONE && d.gate_act != F8_ACT_SIGMOID && d.gate_act != F8_ACT_TANH)
        return f8_set_error(F8_ERR_UNSUPPORTED, "gate_act must be F8_ACT_NONE, F8_ACT_SIGMOID or F8_ACT_TANH");
    if ((d.post_norm == F8_NORM_NONE && (post_w || post_b)) || (d.pre_norm == F8_NORM_NONE && (pre_w || pre_b)))
        return f8_set_error(F8_ERR_UNSUPPORTED, "weights of a norm that is F8_NORM_NONE");
    if (!(d.eps >= 0.f) || !isfinite(d.eps) || !isfinite(d.weight_offset) || !isfinite(d.branch_scale))
        return f8_set_error(F8_ERR_SHAPE, "eps must be finite and not negative, weight_offset and branch_scale finite");
    if (gate && d.gate_rows != 1 && d.gate_rows != d.n) return f8_set_error(F8_ERR_SHAPE, "gate_rows must be 1 or n");
    if (!row_distance(&d.ldx, d.c, d.n) || !row_distance(&d.ldg, d.c, d.n) || !row_distance(&d.ldr, d.c, d.n) || !row_distance(&d.lds, d.c, d.n) ||
        !row_distance(&d.ldy, d.c, d.n) || !row_distance(&d.ldq, d.c, d.n))
        return f8_set_error(F8_ERR_SHAPE, "a row distance is smaller than the row, or too large");
    if (d.n == 0) return F8_OK;
    if (!x || (!q && !y && !residual_out) || (q && !scale) || (!q && scale))
        return f8_set_error(F8_ERR_NULL, "x, and an output (q with scale, y or residual_out), must not be NULL");
    const int ws = real_size(d.w_dtype);
    if (misaligned(x, size) || misaligned(gate, size) || misaligned(residual, size) || misaligned(residual_out, size) || misaligned(y, size) ||
        misaligned(post_w, ws) || misaligned(post_b, ws) || misaligned(pre_w, ws) || misaligned(pre_b, ws) || misaligned(scale, 4))
        return f8_set_error(F8_ERR_ALIGN, "a pointer is not aligned to its element");
    if (f8_pending_timeout() != F8_OK) return F8_ERR_TIMEOUT;
    NormParams p = {d.c, d.post_norm, d.pre_norm, d.gate_act, d.eps, d.weight_offset, d.branch_scale, d.ldx, d.gate_rows == 1 ? 0 : d.ldg,
                    d.ldr, d.lds, d.ldy, d.ldq, x, gate, residual, post_w, post_b, pre_w, pre_b, residual_out, q, scale, y};
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    const bool w32 = d.w_dtype == F8_F32;
    const cudaError_t e = d.dtype == F8_F32   ? launch_norm<float>(p, d.n, true, st)
                          : d.dtype == F8_F16 ? launch_norm<__half>(p, d.n, w32, st)
                                              : launch_norm<__nv_bfloat16>(p, d.n, w32, st);
    if (e != cudaSuccess) return f8_set_error(F8_ERR_CUDA, cudaGetErrorString(e));
    return F8_OK;
}

}   // extern "C"
