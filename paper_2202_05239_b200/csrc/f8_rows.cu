// Rows of real values to 8-bit codes with one scale per row (f8_quantize_rows): gated activations in front of a product, and weight
// matrices, whose rows are output channels.
//
//     v = act(x) * u;   a = max |v|;  s = a / 127;  i = 127 / a;  q = floor(v * i + 1/2)
//
// Bound by memory traffic: every element is read and written once.  Rows of up to 16384 elements stay in registers, 16 elements a
// thread, a warp to 32 warps a row, while the next row is on its way; longer ones take a kernel that reads the row
// twice, the second time from the caches.
// 4096 x 8192 bf16, gate and value with silu, codes alone: 32.6 us, 5.1 TB/s; with the values too 38.1. The forms that few calls take are far from
// that: tensors whose rows lie differently against 16 bytes (halves of a tensor 2 x 8190 wide), element by element, 88.7 and 102 us; 32-bit rows of more
// than 12288 elements with a gate, whose next row finds no room in shared memory, 78.7 us at 2048 x 16384 (2048 x 12288: 41.9); rows of any length
// 364 us at 2048 x 28672 bf16, gated (the activation is computed twice, one element a load), 84 at 2048 x 20000 float.
#include "f8_rowdeal.cuh"

namespace {

struct RowsParams {
    int c, act;
    long long ldx, ldu, ldy, ldq;
    const void *x, *u;
    int8_t *q;
    float *scale;
    void *y;
};

template <typename T, int ACT>
__global__ void __launch_bounds__(ROW_THREADS) long_quantize_kernel(RowsParams p) {
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

// Two values at once.  SiLU of 16-bit rows: v / (1 + exp(-v)) = (v / 4) / (1/4 + exp(-v) / 4) with the exponential and the reciprocal of the
// special function units, each within 2^-22.  -v log2(e) is rounded to t, which alone would put the exponential off by |v| 2^-24; what the
// rounding left out comes from a multiply-add, exactly, and goes in to first order: exp(-v) = 2^t (1 - left ln 2).  The quarter keeps the
// reciprocal above the smallest normal number wherever exp(-v) is finite, as in the plain form (v > -88.7); an infinite one gives 0.
// 4096 x 8192 bf16, gated, codes and values, the same buffers again and again: 38.2 us, with expf and a division 50.2, with the fast exponential and
// quotient 38.7 (42.7 and 42.2 on new buffers each time); codes alone 32.8, 44.9 and 33.5.
template <typename T>
__device__ __forceinline__ F2 activate_two(F2 v, int act) {
    const float2 f = halves(v);
    if (sizeof(T) == 2 && act == F8_ACT_SILU) {
        // beyond these bounds exp(-v) is infinite, or nothing beside 1; kept from the products, which must stay finite
        const F2 w = pair(fminf(fmaxf(f.x, -126.f), 126.f), fminf(fmaxf(f.y, -126.f), 126.f));
        const F2 t = mul2(w, both(-1.44269502f));                                  // log2(e) = 1.44269502 + 1.92596303e-8
        const F2 left = fma2(w, both(1.92596303e-8f), fma2(w, both(1.44269502f), t));
        const float2 e = halves(t);
        const float2 d = halves(fma2(pair(exp2_fast(e.x), exp2_fast(e.y)), fma2(left, both(-0.173286796f), both(0.25f)), both(0.25f)));      // ln(2) / 4
        return mul2(mul2(v, both(0.25f)), pair(reciprocal_fast(d.x), reciprocal_fast(d.y)));
    }
    if (act == F8_ACT_SILU) return pair(activate<F8_ACT_SILU>(f.x), activate<F8_ACT_SILU>(f.y));
    return pair(activate<F8_ACT_GELU>(f.x), activate<F8_ACT_GELU>(f.y));
}

template <typename T, bool ACT, RowMode MODE, int THREADS, int E, bool PIPE>
__global__ void __launch_bounds__(row_block(THREADS), row_blocks(THREADS)) row_quantize_kernel(RowsParams p, long long n) {
    wait_for_stream();
    let_stream_go_on();
    extern __shared__ uint4 smem[];
    __shared__ uint32_t room[2][32];
    using D = Deal<T, MODE, THREADS, E>;
    constexpr int PER = D::PER, PAIRS = D::PAIRS;
    const uint32_t step = gridDim.x * (THREADS == 32 ? 4 : 1), rows = (uint32_t)n;
    uint32_t row = THREADS == 32 ? (threadIdx.x >> 5) * gridDim.x + blockIdx.x : blockIdx.x;
    const uint32_t bx = (uint32_t)p.ldx * sizeof(T), bu = (uint32_t)p.ldu * sizeof(T), by = (uint32_t)p.ldy * sizeof(T), bq = (uint32_t)p.ldq;
    const D d(row_at((const T *)p.x, row, bx), p.c);
    const Ring<row_block(THREADS), PER> ring(smem, p.u ? 2 : 1);
    auto send = [&](uint32_t r, int stage) {
        if (r < rows) {
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                d.send(row_at((const T *)p.x, r, bx), j, ring.place(stage, 0, j));
                if (p.u) d.send(row_at((const T *)p.u, r, bu), j, ring.place(stage, 1, j));
            }
        }
        ring_commit();
    };
    if (PIPE) {
        ring.clear(d);
        send(row, 0);
    }
    for (int stage = 0; row < rows; row += step, stage ^= 1) {
        if (PIPE) {
            send(row + step, stage ^ 1);
            ring_wait();
        }
        F2 v[PER][PAIRS];
        uint4 ru[PER];
        float peak = 0.f;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            unpack<T>(PIPE ? d.take(j, ring.place(stage, 0, j)) : d.load(row_at((const T *)p.x, row, bx), j), v[j]);
            if (!PIPE && p.u) ru[j] = d.load(row_at((const T *)p.u, row, bu), j);
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            if (ACT) {
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) v[j][i] = activate_two<T>(v[j][i], p.act);
            }
            if (p.u) {
                F2 f[PAIRS];
                unpack<T>(PIPE ? d.take(j, ring.place(stage, 1, j)) : ru[j], f);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) v[j][i] = mul2(v[j][i], f[i]);
            }
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) peak = peak_of(peak, v[j][i]);
        }
        T *y = p.y ? row_at((T *)p.y, row, by) : nullptr;
        if (!p.q) {
#pragma unroll
            for (int j = 0; j < PER; ++j) d.store(y, j, v[j]);
            continue;
        }
        const uint32_t top[1] = {block_reduce<THREADS>(magnitude(peak), UMaxOp(), room[stage])};
        RowScale scales[1];
        RowScale::of_warp(top, scales);
        const RowScale &s = scales[0];
        if ((THREADS == 32 ? threadIdx.x & 31 : threadIdx.x) == 0) p.scale[row] = s.scale;
        emit<T>(d, v, s, top[0] < 0x7f800000u, row_at(p.q, row, bq), y);
    }
}

template <typename T, bool ACT, RowMode MODE, int THREADS>
cudaError_t launch_row_quantize_at(const RowsParams &p, long long n, cudaStream_t st) {
    constexpr int PER = ROW_E * (int)sizeof(T) / 16;
    const int tensors = p.u ? 2 : 1;
    if (MODE != LOOSE && ring_bytes(THREADS, PER, tensors) <= RING_MOST)
        return launch_ring<row_quantize_kernel<T, ACT, MODE, THREADS, ROW_E, MODE != LOOSE>>(THREADS, PER, tensors, n, st, p);
    return launch_ring<row_quantize_kernel<T, ACT, LOOSE, THREADS, ROW_E, false>>(THREADS, PER, 0, n, st, p);
}
template <typename T, bool ACT, RowMode MODE>
cudaError_t launch_row_quantize(const RowsParams &p, long long n, cudaStream_t st) {
    const int need = p.c + (MODE == SHIFT ? 16 / (int)sizeof(T) - 1 : 0);
    // As few threads as hold the row, in steps of a quarter and a half between powers of two: threads beyond a row's end cost as much as
    // the others.  Codes alone of 16 M elements, so and with powers of two only (us): rows of 1030 float 17.0 / 22.8, 1536 bf16 7.3 / 9.0, 2047
    // float 14.9 / 23.7, 2304 bf16 8.5 / 11.5, 5000 bf16 9.0 / 11.8, 6000 float 10.7 / 12.8, 8191 bf16 13.8 / 20.5, 11008 bf16 9.7 / 11.6.
    if (need <= 32 * ROW_E) return launch_row_quantize_at<T, ACT, MODE, 32>(p, n, st);
    if (need <= 64 * ROW_E) return launch_row_quantize_at<T, ACT, MODE, 64>(p, n, st);
    if (need <= 96 * ROW_E) return launch_row_quantize_at<T, ACT, MODE, 96>(p, n, st);
    if (need <= 128 * ROW_E) return launch_row_quantize_at<T, ACT, MODE, 128>(p, n, st);
    if (need <= 160 * ROW_E) return launch_row_quantize_at<T, ACT, MODE, 160>(p, n, st);
    if (need <= 192 * ROW_E) return launch_row_quantize_at<T, ACT, MODE, 192>(p, n, st);
    if (need <= 256 * ROW_E) return launch_row_quantize_at<T, ACT, MODE, 256>(p, n, st);
    if (need <= 320 * ROW_E) return launch_row_quantize_at<T, ACT, MODE, 320>(p, n, st);
    if (need <= 384 * ROW_E) return launch_row_quantize_at<T, ACT, MODE, 384>(p, n, st);
    if (need <= 512 * ROW_E) return launch_row_quantize_at<T, ACT, MODE, 512>(p, n, st);
    if (need <= 640 * ROW_E) return launch_row_quantize_at<T, ACT, MODE, 640>(p, n, st);
    if (need <= 768 * ROW_E) return launch_row_quantize_at<T, ACT, MODE, 768>(p, n, st);
    return launch_row_quantize_at<T, ACT, MODE, 1024>(p, n, st);
}

template <typename T, bool ACT>
cudaError_t launch_rows_act(const RowsParams &p, long long n, cudaStream_t st) {
    constexpr int VEC = 16 / sizeof(T);
    RowLayout l(n, sizeof(T), p.c);
    l.add(p.x, p.ldx, sizeof(T));
    l.add(p.u, p.ldu, sizeof(T));
    l.add(p.y, p.ldy, sizeof(T));
    l.add(p.q, p.ldq, 1);
    if (l.same && !l.shift()) return launch_row_quantize<T, ACT, PLAIN>(p, n, st);
    if (l.same && p.c + VEC - 1 <= ROW_MOST) return launch_row_quantize<T, ACT, SHIFT>(p, n, st);
    return launch_row_quantize<T, ACT, LOOSE>(p, n, st);
}
template <typename T>
cudaError_t launch_rows(const RowsParams &p, long long n, cudaStream_t st) {
    if (p.c <= ROW_MOST && std::max({p.ldx, p.ldu, p.ldy, p.ldq}) * (long long)sizeof(T) < (1ll << 32)) return p.act == F8_ACT_NONE ? launch_rows_act<T, false>(p, n, st) : launch_rows_act<T, true>(p, n, st);
    const dim3 grid((unsigned)n);
    switch (p.act) {
        case F8_ACT_SILU: return launch_early(long_quantize_kernel<T, F8_ACT_SILU>, grid, ROW_THREADS, 0, st, p);
        case F8_ACT_GELU: return launch_early(long_quantize_kernel<T, F8_ACT_GELU>, grid, ROW_THREADS, 0, st, p);
        default: return launch_early(long_quantize_kernel<T, F8_ACT_NONE>, grid, ROW_THREADS, 0, st, p);
    }
}

}   // namespace

extern "C" {

f8_status f8_quantize_rows(const f8_rows_desc *desc, const void *x, const void *u, int8_t *q, float *scale, void *y, void *cuda_stream) {
    if (!desc) return f8_set_error(F8_ERR_NULL, "descriptor is NULL");
    f8_rows_desc d = *desc;
    if (d.n < 0 || d.n > 0x7fffffffll || d.c <= 0 || d.c > MOST_EXTENT) return f8_set_error(F8_ERR_SHAPE, "n in 0 .. 2^31 - 1 and c in 1 .. 2^31 - 256 are needed");
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

}   // extern "C"
