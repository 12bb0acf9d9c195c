// Real-valued rows: element types, block-wide reductions and the rounding of a row to 8-bit codes with one scale, shared by the
// kernels around 8-bit products.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "f8_internal.h"

namespace {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Two 32-bit floats in a register pair: this GPU adds and multiplies both in one instruction.
typedef unsigned long long F2;
__device__ __forceinline__ F2 pair(float a, float b) { F2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float2 halves(F2 p) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p)); return r; }
__device__ __forceinline__ F2 add2(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ F2 mul2(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ F2 fma2_down(F2 a, F2 b, F2 c) { F2 r; asm("fma.rm.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ F2 both(float a) { return pair(a, a); }

// The special function units' 2^v and 1 / v, within 2^-22; numbers below the smallest normal one count as 0.
__device__ __forceinline__ float exp2_fast(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
__device__ __forceinline__ float reciprocal_fast(float v) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }

struct SumOp { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
struct UMaxOp { __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; } };

// One value of a whole warp / block, the same in every thread and in every run (fixed order).  `room`: 32 words of shared memory that
// no other reduction of the kernel uses within two barriers.
__device__ __forceinline__ uint32_t warp_reduce(uint32_t v, UMaxOp) { return __reduce_max_sync(0xffffffffu, v); }
template <typename V, typename Op>
__device__ __forceinline__ V warp_reduce(V v, Op op) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
template <int THREADS, typename V, typename Op>
__device__ __forceinline__ V block_reduce(V v, Op op, V *room) {
    v = warp_reduce(v, op);
    if (THREADS == 32) return v;
    constexpr int WARPS = THREADS / 32;
    if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = v;
    __syncthreads();
    if (WARPS <= 8 || (WARPS & (WARPS - 1)) != 0) {
        v = room[0];
#pragma unroll
        for (int w = 1; w < WARPS; ++w) v = op(v, room[w]);
    } else {
        v = room[threadIdx.x & (WARPS - 1)];
#pragma unroll
        for (int d = WARPS / 2; d > 0; d >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, d));
    }
    return v;
}

// The bits of |v|: their order as unsigned numbers is the order of the magnitudes, with infinity above all numbers and NaN
// above infinity, so a maximum over them (unlike one over floats) keeps what is not finite.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Scale of a row's codes and the factor that takes values to codes, from the largest magnitude.
struct RowScale {
    float scale, inverse;
    __device__ __forceinline__ explicit RowScale(uint32_t peak) {
        const float a = __uint_as_float(peak);
        const bool zeros = a < 0x1p-100f, finite = peak < 0x7f800000u;
        scale = zeros ? 0.f : __fdiv_rn(a, 127.f);
        inverse = zeros || !finite ? 0.f : __fdiv_rn(127.f, a);
    }
    // The same for a whole warp that holds the peaks of one or two rows: one division, each quotient by lanes of its own.
    template <int R>
    static __device__ __forceinline__ void of_warp(const uint32_t (&peak)[R], RowScale (&s)[R]) {
        const float a = __uint_as_float(R == 2 && (threadIdx.x & 2) ? peak[R - 1] : peak[0]);
        const bool odd = threadIdx.x & 1;
        const float q = __fdiv_rn(odd ? 127.f : a, odd ? a : 127.f);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool zeros = peak[r] < __float_as_uint(0x1p-100f);
            s[r].scale = __shfl_sync(0xffffffffu, q, 2 * r);
            s[r].inverse = __shfl_sync(0xffffffffu, q, 2 * r + 1);
            if (zeros) s[r].scale = 0.f;
            if (zeros || peak[r] >= 0x7f800000u) s[r].inverse = 0.f;
        }
    }
    __device__ __forceinline__ RowScale() {}
    // floor(v * inverse + 1/2): the sum is rounded towards -infinity, which no integer lies under, so the floor is that of the exact
    // sum.  |v * inverse| <= 127 (1 + 2^-23), hence |code| <= 127 without a clip.  NaN (from 0 * infinity) converts to 0.
    __device__ __forceinline__ int code(float v) const { return __float2int_rd(__fmaf_rd(v, inverse, 0.5f)); }
};

// Longest extent of a row: the loops over rows of any length count in 32 bits, up to a block's step beyond the last element.
constexpr int MOST_EXTENT = 0x7fffff00;

inline int real_size(int dtype) { return dtype == F8_F32 ? 4 : (dtype == F8_F16 || dtype == F8_BF16 ? 2 : 0); }

// Launch whose blocks may start while what is before them in the stream drains; the kernels wait before they touch memory.
template <typename... P, typename... A>
cudaError_t launch_early(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}
__device__ __forceinline__ void wait_for_stream() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_stream_go_on() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

}   // namespace
