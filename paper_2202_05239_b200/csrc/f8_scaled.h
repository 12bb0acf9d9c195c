// Parameters and the arithmetic behind the sums of f8_linear_scaled, shared by its kernels.
#pragma once

#include "f8_real.cuh"

struct ScaledParams {
    int n, k, out;
    int y_dtype, bias_dtype;
    int x_scales, w_scales;
    long long ldx, ldw, ldy;
    const uint8_t *x, *w;
    const float *xs, *ws;
    const void *bias;
    void *y;
};

// Tensor-core kernels (f8_scaled_tc.cu).  cudaErrorNotSupported: an operand lies where bulk tensor copies cannot fetch it.
cudaError_t f8_scaled_tc_launch(const ScaledParams &p, bool x_signed, int *status_word, cudaStream_t st);

namespace {

__device__ __forceinline__ float load_real(const void *p, int dtype, long long i) {
    return dtype == F8_F32 ? ((const float *)p)[i] : dtype == F8_F16 ? to_float(((const __half *)p)[i]) : to_float(((const __nv_bfloat16 *)p)[i]);
}
__device__ __forceinline__ void store_real(void *p, int dtype, long long i, float v) {
    if (dtype == F8_F32) ((float *)p)[i] = v;
    else if (dtype == F8_F16) ((__half *)p)[i] = from_float<__half>(v);
    else ((__nv_bfloat16 *)p)[i] = from_float<__nv_bfloat16>(v);
}
__device__ __forceinline__ float scaled(int acc, float sx, float sw, float b) { return __fmaf_rn(__fmul_rn(__int2float_rn(acc), sx), sw, b); }

// Four neighbouring outputs from their sums; `wide`: y may be written in words of four elements here.
__device__ __forceinline__ void store_scaled4(const ScaledParams &p, const int (&acc)[4], int m, int o, float sx, const float (&sw)[4], const float (&b)[4], bool wide) {
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = scaled(acc[k], sx, sw[k], b[k]);
    const long long at = (long long)m * p.ldy + o;
    if (wide) {
        if (p.y_dtype == F8_F32) {
            *(float4 *)((float *)p.y + at) = make_float4(v[0], v[1], v[2], v[3]);
        } else if (p.y_dtype == F8_F16) {
            const __half2 a = __floats2half2_rn(v[0], v[1]), c = __floats2half2_rn(v[2], v[3]);
            *(uint2 *)((__half *)p.y + at) = make_uint2(*(const uint32_t *)&a, *(const uint32_t *)&c);
        } else {
            const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), c = __floats2bfloat162_rn(v[2], v[3]);
            *(uint2 *)((__nv_bfloat16 *)p.y + at) = make_uint2(*(const uint32_t *)&a, *(const uint32_t *)&c);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (o + k < p.out) store_real(p.y, p.y_dtype, at + k, v[k]);
    }
}

}   // namespace
