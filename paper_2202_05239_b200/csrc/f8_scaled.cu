// y = x w^T of 8-bit codes with one real scale per row of x and one per row of w:
//
//     acc = sum_k x[i, k] w[j, k]   (exact, int32);     y[i, j] = round( fma((float)acc * sx[i], sw[j], b[j]) )
//
// The tensor-core kernels (f8_scaled_tc.cu) fetch operands whose rows start at multiples of 16 bytes.  The kernel here takes every
// alignment and row distance: tiles of 64 x 64 on mma.sync m16n8k32, K in chunks of 64 bytes through
// padded rows of shared memory, the next chunk on its way in registers while one is multiplied.
#include <math.h>

#include <algorithm>

#include "f8_scaled.h"

namespace {

// 16 bytes from `p`, those from `valid` on as zeros.  ALIGNED: p is a multiple of 16.  Otherwise the one or two 16-byte granules that
// hold wanted bytes are read whole and shifted together; a granule that holds one byte of an allocation lies within its page.
template <bool ALIGNED>
__device__ __forceinline__ uint4 load_bytes(const uint8_t *p, int valid) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (valid <= 0) return v;
    if (ALIGNED) {
        v = *(const uint4 *)p;
    } else {
        const uint32_t sh = (uint32_t)(uintptr_t)p & 15u;
        const uint4 *g = (const uint4 *)(p - sh);
        uint4 a = g[0], b = make_uint4(0, 0, 0, 0);
        if (valid + (int)sh > 16) b = g[1];
        // by words, then by bytes
        if (sh & 8u) { a.x = a.z; a.y = a.w; a.z = b.x; a.w = b.y; b.x = b.z; b.y = b.w; }
        if (sh & 4u) { a.x = a.y; a.y = a.z; a.z = a.w; a.w = b.x; b.x = b.y; }
        const uint32_t bits = (sh & 3u) * 8u;
        v = make_uint4(__funnelshift_r(a.x, a.y, bits), __funnelshift_r(a.y, a.z, bits), __funnelshift_r(a.z, a.w, bits), __funnelshift_r(a.w, b.x, bits));
    }
    if (valid < 16) {
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int n = valid - 4 * j;
            w[j] = n >= 4 ? w[j] : n <= 0 ? 0u : w[j] & (0xffffffffu >> (32 - 8 * n));
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return v;
}

template <bool SIGNED>
__device__ __forceinline__ void mma_16x8x32(int (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (SIGNED)
        asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

constexpr int GT = 64, GK = 64, GROW = GK + 16, G_THREADS = 128;     // rows of 80 bytes: the eight rows of a fragment fall on different banks

template <bool SIGNED, bool ALIGNED>
__global__ void __launch_bounds__(G_THREADS) scaled_any_kernel(ScaledParams p) {
    wait_for_stream();
    let_stream_go_on();
    __shared__ __align__(16) uint8_t sm[2][2][GT * GROW];
    const int m0 = blockIdx.y * GT, n0 = blockIdx.x * GT;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int wm = (warp >> 1) * 32, wn = (warp & 1) * 32;
    int acc[2][4][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[i][j][k] = 0;
    // two 16-byte pieces of each operand per thread and chunk
    uint4 next[2][2];
    auto fetch = [&](int k0) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int piece = threadIdx.x + G_THREADS * h, row = piece >> 2, kk = k0 + 16 * (piece & 3);
            next[0][h] = load_bytes<ALIGNED>(p.x + (long long)(m0 + row) * p.ldx + kk, m0 + row < p.n ? p.k - kk : 0);
            next[1][h] = load_bytes<ALIGNED>(p.w + (long long)(n0 + row) * p.ldw + kk, n0 + row < p.out ? p.k - kk : 0);
        }
    };
    auto keep = [&](int buf) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int piece = threadIdx.x + G_THREADS * h, at = (piece >> 2) * GROW + 16 * (piece & 3);
            *(uint4 *)&sm[buf][0][at] = next[0][h];
            *(uint4 *)&sm[buf][1][at] = next[1][h];
        }
    };
    fetch(0);
    keep(0);
    __syncthreads();
    int buf = 0;
    for (int k0 = 0; k0 < p.k; k0 += GK, buf ^= 1) {
        const bool more = k0 + GK < p.k;
        if (more) fetch(k0 + GK);
        const uint8_t *A = sm[buf][0], *B = sm[buf][1];
#pragma unroll
        for (int ks = 0; ks < GK; ks += 32) {
            uint32_t a[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint8_t *r = A + (wm + 16 * i + g) * GROW + ks + 4 * t;
                a[i][0] = *(const uint32_t *)r;
                a[i][1] = *(const uint32_t *)(r + 8 * GROW);
                a[i][2] = *(const uint32_t *)(r + 16);
                a[i][3] = *(const uint32_t *)(r + 8 * GROW + 16);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint8_t *r = B + (wn + 8 * j + g) * GROW + ks + 4 * t;
                const uint32_t b0 = *(const uint32_t *)r, b1 = *(const uint32_t *)(r + 16);
#pragma unroll
                for (int i = 0; i < 2; ++i) mma_16x8x32<SIGNED>(acc[i][j], a[i], b0, b1);
            }
        }
        if (more) keep(buf ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int m = m0 + wm + 16 * i + 8 * h + g;
            if (m >= p.n) continue;
            const float sx = p.xs[p.x_scales == 1 ? 0 : m];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int o = n0 + wn + 8 * j + 2 * t + k;
                    if (o >= p.out) continue;
                    const float b = p.bias ? load_real(p.bias, p.bias_dtype, o) : 0.f;
                    store_real(p.y, p.y_dtype, (long long)m * p.ldy + o, scaled(acc[i][j][2 * h + k], sx, p.ws[p.w_scales == 1 ? 0 : o], b));
                }
        }
}

cudaError_t launch_any(const ScaledParams &p, bool x_signed, cudaStream_t st) {
    const bool aligned = ((((uintptr_t)p.x | (uintptr_t)p.w) & 15) | ((unsigned long long)(p.ldx | p.ldw) & 15)) == 0;
    const long long rows = ((long long)p.n + GT - 1) / GT;
    // blocks of one grid share the rows of x: at most 65535 of them, so very many rows go out as several launches
    for (long long at = 0; at < rows; at += 65535) {
        ScaledParams q = p;
        q.n = (int)std::min<long long>(p.n - at * GT, 65535ll * GT);
        q.x = p.x + at * GT * p.ldx;
        if (p.x_scales != 1) q.xs = p.xs + at * GT;
        q.y = (char *)p.y + at * GT * p.ldy * real_size(p.y_dtype);
        const dim3 grid((unsigned)((p.out + (long long)GT - 1) / GT), (unsigned)((q.n + GT - 1) / GT));
        cudaError_t e;
        if (x_signed) e = aligned ? launch_early(scaled_any_kernel<true, true>, grid, G_THREADS, 0, st, q) : launch_early(scaled_any_kernel<true, false>, grid, G_THREADS, 0, st, q);
        else e = aligned ? launch_early(scaled_any_kernel<false, true>, grid, G_THREADS, 0, st, q) : launch_early(scaled_any_kernel<false, false>, grid, G_THREADS, 0, st, q);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}   // namespace

extern "C" f8_status f8_linear_scaled(const f8_scaled_desc *desc, const void *x, const float *x_scale, const int8_t *w, const float *w_scale,
                                      const void *bias, void *y, void *cuda_stream) {
    if (!desc) return f8_set_error(F8_ERR_NULL, "descriptor is NULL");
    f8_scaled_desc d = *desc;
    if (d.n < 0 || d.k <= 0 || d.out <= 0) return f8_set_error(F8_ERR_SHAPE, "n >= 0, k > 0 and out > 0 are needed");
    if (d.x_dtype != F8_U8 && d.x_dtype != F8_S8) return f8_set_error(F8_ERR_DTYPE, "x_dtype must be F8_U8 or F8_S8");
    const int ys = real_size(d.y_dtype), bs = bias ? real_size(d.bias_dtype) : 1;
    if (!ys || !bs) return f8_set_error(F8_ERR_DTYPE, "y_dtype and bias_dtype must be F8_F32, F8_F16 or F8_BF16");
    if ((long long)d.k * (d.x_dtype == F8_U8 ? 255 : 128) * 128 >= (1ll << 31))
        return f8_set_error(F8_ERR_ACC_BOUND, "k products cannot be guaranteed to fit the int32 accumulator");
    if ((d.x_scales != 1 && d.x_scales != d.n) || (d.w_scales != 1 && d.w_scales != d.out))
        return f8_set_error(F8_ERR_SHAPE, "x_scales must be n or 1, w_scales out or 1");
    if (d.ldx == 0) d.ldx = d.k;
    if (d.ldw == 0) d.ldw = d.k;
    if (d.ldy == 0) d.ldy = d.out;
    const long long most = 1ll << 40;
    if (d.ldx < d.k || d.ldw < d.k || d.ldy < d.out || d.ldx > most || d.ldw > most || d.ldy > most ||
        (d.n > 1 && (d.ldx > (1ll << 50) / d.n || d.ldy > (1ll << 50) / d.n)) || d.ldw > (1ll << 50) / d.out)
        return f8_set_error(F8_ERR_SHAPE, "a row distance is smaller than the row, or too large");
    if (d.n == 0) return F8_OK;
    if (!x || !x_scale || !w || !w_scale || !y) return f8_set_error(F8_ERR_NULL, "x, w, their scales and y must not be NULL");
    if ((((uintptr_t)x_scale | (uintptr_t)w_scale) & 3) || ((uintptr_t)y & (uintptr_t)(ys - 1)) || ((uintptr_t)bias & (uintptr_t)(bs - 1)))
        return f8_set_error(F8_ERR_ALIGN, "a pointer is not aligned to its element");
    if (f8_pending_timeout() != F8_OK) return F8_ERR_TIMEOUT;
    const ScaledParams p = {d.n, d.k, d.out, d.y_dtype, d.bias_dtype, d.x_scales, d.w_scales, d.ldx, d.ldw, d.ldy, (const uint8_t *)x,
                            (const uint8_t *)w, x_scale, w_scale, bias, y};
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = f8_force_direct() ? cudaErrorNotSupported : f8_scaled_tc_launch(p, d.x_dtype == F8_S8, f8_status_word(), st);
    if (e == cudaErrorNotSupported) e = launch_any(p, d.x_dtype == F8_S8, st);
    if (e != cudaSuccess) return f8_set_error(F8_ERR_CUDA, cudaGetErrorString(e));
    return F8_OK;
}
