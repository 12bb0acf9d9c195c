// Log probabilities of given tokens, entropy and the largest alternatives of rows of logits (32-bit codes of a network, or real
// values):  with m the largest logit of a row, d_j = (m - l_j) * c >= 0 (c the inverse temperature, times 2^-fl for codes) and
// r = the sum of exp(-d_j) over all j but the first largest one,
//
//     log p_j = -d_j - log(1 + r)          H = log(1 + r) + sum_j d_j exp(-d_j) / (1 + r)
//
// Leaving the largest term (exactly 1) out of the sum keeps the relative precision of rows whose largest logit has nearly all the
// probability: log1p(r) of a small r instead of the logarithm of a sum next to 1, and two terms of one sign.  Differences of
// codes are taken as integers, so codes beyond 2^24 lose nothing.
//
// Bound by reading the logits once.
#include <math.h>

#include "f8_real.cuh"

namespace {

constexpr int LP_THREADS = 256;

struct LpParams {
    int v, tokens, top;
    float c;
    long long ldl;
    const void *logits;
    const int64_t *ids;
    float *lp, *entropy, *top_lp;
    int64_t *top_ids;
};

// Logits as unsigned numbers of the same order: NaN above +infinity, both zeros equal.
__device__ __forceinline__ uint32_t order_of(float v) {
    if (v != v) return 0xffffffffu;
    const uint32_t b = __float_as_uint(v + 0.f);
    return (int)b < 0 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float((int)o < 0 ? o & 0x7fffffffu : ~o); }

template <typename T> struct Logit {        // real logits
    static __device__ __forceinline__ uint32_t order(T l) { return order_of(to_float(l)); }
    // what the largest one lacks of c times the distance, from the orders of both
    static __device__ __forceinline__ float distance(uint32_t top, uint32_t o, float c) { return (value_of(top) - value_of(o)) * c; }
    static __device__ __forceinline__ bool bad(uint32_t top) { return top >= 0xff800000u; }       // +infinity or NaN
    static __device__ __forceinline__ bool empty(uint32_t top) { return top == 0x007fffffu; }     // -infinity
};
template <> struct Logit<int> {             // codes
    static __device__ __forceinline__ uint32_t order(int l) { return (uint32_t)l ^ 0x80000000u; }
    static __device__ __forceinline__ float distance(uint32_t top, uint32_t o, float c) { return (float)(top - o) * c; }
    static __device__ __forceinline__ bool bad(uint32_t) { return false; }
    static __device__ __forceinline__ bool empty(uint32_t) { return false; }
};

struct MaxOp { __device__ __forceinline__ unsigned long long operator()(unsigned long long a, unsigned long long b) const { return a > b ? a : b; } };

template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_kernel(LpParams p) {
    wait_for_stream();
    let_stream_go_on();
    __shared__ unsigned long long room[32];
    __shared__ float froom[32];
    const long long row = blockIdx.x;
    const T *l = (const T *)p.logits + row * p.ldl;
    // order and index in one number: the larger logit first, then the smaller index
    auto key = [&](int j) { return (unsigned long long)Logit<T>::order(l[j]) << 32 | (uint32_t)~j; };
    unsigned long long best = 0;
    for (int j = threadIdx.x; j < p.v; j += LP_THREADS) best = max(best, key(j));
    best = block_reduce<LP_THREADS>(best, MaxOp(), room);
    const uint32_t top = (uint32_t)(best >> 32);
    const bool bad = Logit<T>::bad(top), empty = Logit<T>::empty(top);
    float r = 0.f, t = 0.f;
    for (int j = threadIdx.x; j < p.v; j += LP_THREADS) {
        const float d = Logit<T>::distance(top, Logit<T>::order(l[j]), p.c), e = expf(-d);
        if (j != (int)~(uint32_t)best) r += e;
        if (e > 0.f) t += e * d;
    }
    r = block_reduce<LP_THREADS>(r, SumOp(), froom);
    __syncthreads();
    t = block_reduce<LP_THREADS>(t, SumOp(), froom);
    const float lse = log1pf(r);
    auto logprob = [&](uint32_t o) { return bad ? __int_as_float(0x7fffffff) : empty ? -INFINITY : -Logit<T>::distance(top, o, p.c) - lse; };
    if (threadIdx.x == 0 && p.entropy) p.entropy[row] = bad ? __int_as_float(0x7fffffff) : empty ? 0.f : lse + t / (1.f + r);
    if (p.lp)
        for (int i = threadIdx.x; i < p.tokens; i += LP_THREADS) {
            const int64_t id = p.ids[row * p.tokens + i];
            p.lp[row * p.tokens + i] = id < 0 ? 0.f : id >= p.v ? __int_as_float(0x7fffffff) : logprob(Logit<T>::order(l[id]));
        }
    for (int i = 0; i < p.top; ++i) {
        if (threadIdx.x == 0) {
            if (p.top_lp) p.top_lp[row * p.top + i] = logprob((uint32_t)(best >> 32));
            if (p.top_ids) p.top_ids[row * p.top + i] = (int64_t)~(uint32_t)best;
        }
        if (i + 1 == p.top) break;
        unsigned long long next = 0;
        for (int j = threadIdx.x; j < p.v; j += LP_THREADS) {
            const unsigned long long k = key(j);
            if (k < best) next = max(next, k);
        }
        __syncthreads();
        best = block_reduce<LP_THREADS>(next, MaxOp(), room);
    }
}

}   // namespace

extern "C" f8_status f8_token_logprobs(const f8_logprobs_desc *desc, const void *logits, const int64_t *tokens, float *logprobs, float *entropy,
                                       float *top_logprobs, int64_t *top_ids, void *cuda_stream) {
    if (!desc) return f8_set_error(F8_ERR_NULL, "descriptor is NULL");
    f8_logprobs_desc d = *desc;
    if (d.n < 0 || d.n > 0x7fffffffll || d.v <= 0 || d.tokens < 0) return f8_set_error(F8_ERR_SHAPE, "n in 0 .. 2^31 - 1, v > 0 and tokens >= 0 are needed");
    if (d.top < 0 || d.top > 32 || d.top > d.v) return f8_set_error(F8_ERR_SHAPE, "top must be in 0 .. 32 and at most v");
    if (!(d.inv_temperature > 0.f) || !isfinite(d.inv_temperature)) return f8_set_error(F8_ERR_SHAPE, "inv_temperature must be positive and finite");
    const int size = d.dtype == F8_S32 ? 4 : real_size(d.dtype);
    if (!size) return f8_set_error(F8_ERR_DTYPE, "dtype must be F8_S32, F8_F32, F8_F16 or F8_BF16");
    if (d.dtype == F8_S32 && (d.fl < -8 || d.fl > 32)) return f8_set_error(F8_ERR_FL_RANGE, "fl outside [-8, 32]");
    const float c = d.dtype == F8_S32 ? ldexpf(d.inv_temperature, -d.fl) : d.inv_temperature;
    if (!(c > 0.f) || !isfinite(c)) return f8_set_error(F8_ERR_SHAPE, "inv_temperature * 2^-fl leaves the range of 32-bit floats");
    if (d.ldl == 0) d.ldl = d.v;
    if (d.ldl < d.v || d.ldl > (1ll << 40) || (d.n > 1 && d.ldl > (1ll << 50) / d.n))
        return f8_set_error(F8_ERR_SHAPE, "the row distance is smaller than the row, or too large");
    if (d.n == 0) return F8_OK;
    if (!logits || (logprobs && d.tokens && !tokens)) return f8_set_error(F8_ERR_NULL, "logits, and tokens where logprobs are asked for, must not be NULL");
    if (!logprobs && !entropy && !((top_logprobs || top_ids) && d.top > 0)) return f8_set_error(F8_ERR_NULL, "no output is asked for");
    if (((uintptr_t)logits & (uintptr_t)(size - 1)) || (((uintptr_t)tokens | (uintptr_t)top_ids) & 7) ||
        (((uintptr_t)logprobs | (uintptr_t)entropy | (uintptr_t)top_logprobs) & 3))
        return f8_set_error(F8_ERR_ALIGN, "a pointer is not aligned to its element");
    if (f8_pending_timeout() != F8_OK) return F8_ERR_TIMEOUT;
    LpParams p = {d.v, d.tokens, top_logprobs || top_ids ? d.top : 0, c, d.ldl, logits, tokens, logprobs, entropy, top_logprobs, top_ids};
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    const dim3 grid((unsigned)d.n);
    cudaError_t e;
    switch (d.dtype) {
        case F8_S32: e = launch_early(logprobs_kernel<int>, grid, LP_THREADS, 0, st, p); break;
        case F8_F32: e = launch_early(logprobs_kernel<float>, grid, LP_THREADS, 0, st, p); break;
        case F8_F16: e = launch_early(logprobs_kernel<__half>, grid, LP_THREADS, 0, st, p); break;
        default: e = launch_early(logprobs_kernel<__nv_bfloat16>, grid, LP_THREADS, 0, st, p); break;
    }
    if (e != cudaSuccess) return f8_set_error(F8_ERR_CUDA, cudaGetErrorString(e));
    return F8_OK;
}
