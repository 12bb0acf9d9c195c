// Rows of real values in registers: how the elements of a row are dealt out to threads, loads and stores of every alignment, the ring
// through which a block fetches the next row while it works on one, rounding to codes.
#pragma once

#include <math.h>

#include <algorithm>
#include <atomic>

#include "f8_real.cuh"

namespace {

constexpr int ROW_THREADS = 256;          // of the kernels for rows of any length
constexpr int ROW_E = 16;                 // elements of a row per thread
constexpr int ROW_MOST = 1024 * ROW_E;    // longest row that stays in registers

template <int ACT>
__device__ __forceinline__ float activate(float v) {
    if (ACT == F8_ACT_SILU) return v / (1.f + expf(-v));
    if (ACT == F8_ACT_GELU) return v * normcdff(v);      // relative precision for negative v too, which 1 + erf loses
    if (ACT == F8_ACT_SIGMOID) return 1.f / (1.f + expf(-v));
    if (ACT == F8_ACT_TANH) return tanhf(v);
    return v;
}

// ------------------------------------------------------------------ rows in registers

// How the elements of a row are dealt out to its threads, in vectors of 16 bytes of the real tensors:
//   PLAIN   all rows of all tensors start at a multiple of 16 bytes and hold whole vectors
//   SHIFT   all tensors start at the same distance m (in elements) behind such a multiple, which may change from row to row, as in
//           dense rows of an odd width: the vectors lie on the multiples of 16 bytes, those at the ends of a row are read whole (a
//           granule of 16 bytes that holds an element of the row) and written element by element
//   LOOSE   anything else: neighbouring threads take neighbouring elements one by one
enum RowMode { PLAIN, SHIFT, LOOSE };

// The row kernels are bound by instruction issue as much as by memory, so they work on pairs throughout.
// the largest magnitude so far and two more; NaN wins
__device__ __forceinline__ float peak_of(float m, F2 p) {
    const float2 f = halves(p);
    asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(fabsf(f.x)), "f"(fabsf(f.y)));
    return m;
}

__device__ __forceinline__ F2 unpack2(uint32_t w, __half) {
    const float2 f = __half22float2(*(const __half2 *)&w);
    return pair(f.x, f.y);
}
__device__ __forceinline__ F2 unpack2(uint32_t w, __nv_bfloat16) { return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack2(F2 p, __half) {
    const float2 f = halves(p);
    const __half2 h = __floats2half2_rn(f.x, f.y);
    return *(const uint32_t *)&h;
}
__device__ __forceinline__ uint32_t pack2(F2 p, __nv_bfloat16) {
    const float2 f = halves(p);
    const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
    return *(const uint32_t *)&h;
}
template <typename T>
__device__ __forceinline__ void unpack(const uint4 &w, F2 (&f)[8 / sizeof(T)]) {
    if constexpr (sizeof(T) == 4) {
        f[0] = pair(__uint_as_float(w.x), __uint_as_float(w.y));
        f[1] = pair(__uint_as_float(w.z), __uint_as_float(w.w));
    } else {
        f[0] = unpack2(w.x, T()); f[1] = unpack2(w.y, T()); f[2] = unpack2(w.z, T()); f[3] = unpack2(w.w, T());
    }
}
template <typename T>
__device__ __forceinline__ uint4 pack(const F2 (&f)[8 / sizeof(T)]) {
    if constexpr (sizeof(T) == 4) {
        const float2 a = halves(f[0]), b = halves(f[1]);
        return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
    } else {
        return make_uint4(pack2(f[0], T()), pack2(f[1], T()), pack2(f[2], T()), pack2(f[3], T()));
    }
}
__device__ __forceinline__ uint32_t bits_of(float v) { return __float_as_uint(v); }
__device__ __forceinline__ uint32_t bits_of(__half v) { return __half_as_ushort(v); }
__device__ __forceinline__ uint32_t bits_of(__nv_bfloat16 v) { return __bfloat16_as_ushort(v); }
// element k of a vector
template <typename T>
__device__ __forceinline__ void set_element(uint4 &w, int k, uint32_t bits) {
    uint32_t *u = &w.x;
    if (sizeof(T) == 4) u[k] = bits;
    else u[k >> 1] = k & 1 ? __byte_perm(u[k >> 1], bits, 0x5410) : __byte_perm(u[k >> 1], bits, 0x3254);
}
template <typename T>
__device__ __forceinline__ T get_element(const uint4 &w, int k) {
    const uint32_t *u = &w.x;
    if constexpr (sizeof(T) == 4) return __uint_as_float(u[k]);
    else {
        const unsigned short b = (unsigned short)(k & 1 ? u[k >> 1] >> 16 : u[k >> 1] & 0xffffu);
        return *(const T *)&b;
    }
}

template <typename T, RowMode MODE, int THREADS, int E>
struct Deal {
    static constexpr int VEC = 16 / sizeof(T), PER = E / VEC, PAIRS = VEC / 2;
    int c, first;
    __device__ __forceinline__ Deal(const void *row, int c_) : c(c_) {
        const int tid = (int)(THREADS == 32 ? threadIdx.x & 31 : threadIdx.x);
        const int m = MODE == SHIFT ? (int)((uintptr_t)row / sizeof(T) % VEC) : 0;
        first = MODE == LOOSE ? tid : tid * VEC - m;
    }
    __device__ __forceinline__ int at(int j, int k) const { return MODE == LOOSE ? first + (j * VEC + k) * THREADS : first + j * THREADS * VEC + k; }
    __device__ __forceinline__ bool on(int j) const { return at(j, 0) < c; }                       // vector j holds an element of the row
    __device__ __forceinline__ bool whole(int j) const { return MODE == PLAIN || (MODE == SHIFT && at(j, 0) >= 0 && at(j, 0) + VEC <= c); }
    __device__ __forceinline__ bool in(int j, int k) const { return MODE == SHIFT ? (unsigned)at(j, k) < (unsigned)c : at(j, MODE == PLAIN ? 0 : k) < c; }

    // Vector j, zero where the row has no element.  The loads stay out of the first-level cache, which the norm weights want, and
    // off the read-only path: what is read may have been written by the grid before while the blocks here already waited.
    __device__ __forceinline__ uint4 load(const T *row, int j) const {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (!on(j)) return w;
        if constexpr (MODE == LOOSE) {
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                if (in(j, k)) set_element<T>(w, k, bits_of(row[at(j, k)]));
        } else {
            asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "l"(row + at(j, 0)) : "memory");
            if (!whole(j)) {
#pragma unroll
                for (int k = 0; k < VEC; ++k)
                    if (!in(j, k)) set_element<T>(w, k, 0u);
            }
        }
        return w;
    }
    // The same in two steps: the vector on its way to this thread's own place in shared memory, and from there.
    __device__ __forceinline__ void send(const T *row, int j, uint32_t place) const {
        if (on(j)) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(place), "l"(row + at(j, 0)) : "memory");
    }
    // (places that nothing is sent to hold zeros, see Ring::clear)
    __device__ __forceinline__ uint4 take(int j, uint32_t place) const {
        uint4 w;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(place) : "memory");
        if (MODE == SHIFT && !whole(j)) {
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                if (!in(j, k)) set_element<T>(w, k, 0u);
        }
        return w;
    }
    __device__ __forceinline__ void store(T *row, int j, const F2 (&f)[PAIRS]) const {
        if (!on(j)) return;
        const uint4 w = pack<T>(f);
        if (whole(j)) {
            *(uint4 *)(row + at(j, 0)) = w;
        } else {
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                if (in(j, k)) row[at(j, k)] = get_element<T>(w, k);
        }
    }
    __device__ __forceinline__ void store_codes(int8_t *row, int j, const uint32_t (&w)[VEC / 4]) const {
        if (!on(j)) return;
        if (whole(j)) {
            if constexpr (VEC == 8) *(uint2 *)(row + at(j, 0)) = make_uint2(w[0], w[1]);
            else *(uint32_t *)(row + at(j, 0)) = w[0];
        } else {
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                if (in(j, k)) row[at(j, k)] = (int8_t)(w[k >> 2] >> (8 * (k & 3)));
        }
    }
    // vector j, on, of c norm weights (32-bit or T) or of a gate that all rows share; zero where the row has no element
    template <bool W32>
    __device__ __forceinline__ void weights(const void *w, int j, F2 (&f)[PAIRS]) const {
        if constexpr (MODE == PLAIN) {
            if constexpr (VEC == 4 || !W32) {
                unpack<T>(*(const uint4 *)((const T *)w + at(j, 0)), f);
            } else {
                const ulonglong2 a = *(const ulonglong2 *)((const float *)w + at(j, 0)), b = *(const ulonglong2 *)((const float *)w + at(j, 0) + 4);
                f[0] = a.x; f[1] = a.y; f[PAIRS - 2] = b.x; f[PAIRS - 1] = b.y;
            }
        } else {
            float e[VEC];
#pragma unroll
            for (int k = 0; k < VEC; ++k) e[k] = !in(j, k) ? 0.f : W32 ? ((const float *)w)[at(j, k)] : to_float(((const T *)w)[at(j, k)]);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) f[i] = pair(e[2 * i], e[2 * i + 1]);
        }
    }
    // zeros where the row has no element
    __device__ __forceinline__ void mask(int j, F2 (&f)[PAIRS]) const {
        if (whole(j) && on(j)) return;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            const float2 v = halves(f[i]);
            f[i] = pair(in(j, 2 * i) ? v.x : 0.f, in(j, 2 * i + 1) ? v.y : 0.f);
        }
    }
};

// Codes, and the values they stand for, of a row whose values are in registers.  v * inverse + 1/2 is added to 3 * 2^14 in one
// multiply-add rounded towards -infinity: the sum's last place is 2^-8, so the second byte of its bits is the floor.  (The sum
// loses places below 2^-8 towards -infinity, which no integer lies under.)
template <typename T, typename D>
__device__ __forceinline__ void emit(const D &d, F2 (&v)[D::PER][D::PAIRS], const RowScale &s, bool finite, int8_t *q, T *y) {
    if (!finite) {          // codes of 0, which the scale makes NaN
#pragma unroll
        for (int j = 0; j < D::PER; ++j)
#pragma unroll
            for (int i = 0; i < D::PAIRS; ++i) v[j][i] = 0ull;
    }
    const F2 inverse = both(s.inverse), place = both(49152.5f), back = both(-49152.f), scale = both(s.scale);
#pragma unroll
    for (int j = 0; j < D::PER; ++j) {
        uint32_t code[D::VEC / 4];
        F2 f[D::PAIRS];
#pragma unroll
        for (int i = 0; i < D::PAIRS; ++i) f[i] = fma2_down(v[j][i], inverse, place);
#pragma unroll
        for (int i = 0; i < D::VEC / 4; ++i) {
            const float2 a = halves(f[2 * i]), b = halves(f[2 * i + 1]);
            code[i] = __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0051),
                                  __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0051), 0x5410);
        }
        d.store_codes(q, j, code);
        if (!y) continue;
#pragma unroll
        for (int i = 0; i < D::PAIRS; ++i) f[i] = mul2(add2(f[i] & 0xffffff00ffffff00ull, back), scale);
        d.store(y, j, f);
    }
}

// Row `row` of a matrix whose rows are `bytes` apart: one multiply-add of two 32-bit numbers (the kernels for rows in registers take
// distances below 2^32 bytes).
template <typename T> __device__ __forceinline__ T *row_at(T *base, uint32_t row, uint32_t bytes) { return (T *)((char *)base + (unsigned long long)row * bytes); }
template <typename T> __device__ __forceinline__ const T *row_at(const T *base, uint32_t row, uint32_t bytes) {
    return (const T *)((const char *)base + (unsigned long long)row * bytes);
}

__host__ __device__ constexpr int row_block(int threads) { return threads == 32 ? 128 : threads; }      // a warp a row: four rows in a block
// blocks of an SM that the registers have to leave room for (64 a thread)
constexpr int row_blocks(int threads) { return 1024 / row_block(threads); }

// Where many rows go through few blocks (PIPE), a block walks rows gridDim apart and has the next one on its way while it works on
// one: the vectors of every thread go to places of its own in shared memory, two rows deep, which takes no barrier between threads.
template <int BLOCK, int PER>
struct Ring {
    uint32_t mine;
    int tensors;
    __device__ __forceinline__ Ring(const void *smem, int tensors_) : mine((uint32_t)__cvta_generic_to_shared(smem) + threadIdx.x * 16u), tensors(tensors_) {}
    // zeros where no row of this block has an element
    template <typename D>
    __device__ __forceinline__ void clear(const D &d) const {
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (!d.on(j))
                for (int i = 0; i < 2 * tensors; ++i)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(mine + (uint32_t)((i * PER + j) * BLOCK * 16)), "r"(0) : "memory");
    }
    __device__ __forceinline__ uint32_t place(int stage, int tensor, int j) const { return mine + (uint32_t)(((stage * tensors + tensor) * PER + j) * BLOCK * 16); }
};
__device__ __forceinline__ void ring_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void ring_wait() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }

// How the tensors of a call lie relative to each other.
struct RowLayout {
    long long n;
    int size, vec;
    bool first = true, same = true, whole = true, near = true;
    uintptr_t base = 0, step = 0;
    RowLayout(long long n_, int size_, int c) : n(n_), size(size_), vec(16 / size_) { whole = c % vec == 0; }
    // a matrix of `bytes` a element and a distance of ld elements between its rows
    void add(const void *p, long long ld, int bytes) {
        if (!p) return;
        const uintptr_t b = (uintptr_t)p / bytes % vec, s = n > 1 ? (uintptr_t)ld % vec : 0;
        if (first) { base = b; step = s; first = false; }
        same = same && b == base && s == step;
        near = near && ld * bytes < (1ll << 32);
    }
    void vector(const void *p) { whole = whole && ((uintptr_t)p & 15) == 0; }
    int shift() const { return base != 0 || step != 0 || !whole; }
};

// As many blocks as the SMs hold at once, or as there are rows.  `tensors`: those whose rows go through the ring (0: none do).
// What the runtime says of a kernel is asked once for each device and size of the ring.
struct RingFit { std::atomic<int> held[64][8]; };
constexpr size_t RING_MOST = 220 * 1024;
inline size_t ring_bytes(int threads, int per, int tensors) { return (size_t)2 * tensors * per * row_block(threads) * 16; }

// Where there are more rows than blocks hold, the blocks are a multiple of eight, so that a block's rows all lie alike (SHIFT).
template <auto KERNEL, typename... A>
cudaError_t launch_ring(int threads, int per, int tensors, long long n, cudaStream_t st, A... a) {
    static RingFit fit;
    const int block = row_block(threads);
    const size_t smem = ring_bytes(threads, per, tensors);
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    int held = fit.held[dev][tensors].load(std::memory_order_relaxed);
    if (held == 0) {
        int sms = 0, blocks = 0;
        const size_t most = RING_MOST;
        e = cudaFuncSetAttribute((const void *)KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, (const void *)KERNEL, block, smem);
        if (e != cudaSuccess) return e;
        held = std::max(std::max(blocks, 1) * sms / 8 * 8, 8);
        fit.held[dev][tensors].store(held, std::memory_order_relaxed);
    }
    const long long blocks = threads == 32 ? (n + 3) / 4 : n;
    return launch_early(KERNEL, dim3((unsigned)std::min<long long>(blocks, held)), block, smem, st, a..., n);
}

// Row distance: 0 stands for dense rows; false where rows would overlap or the matrix would pass what a pointer reaches.
bool row_distance(long long *ld, int c, long long n) {
    if (*ld == 0) *ld = c;
    return *ld >= c && *ld <= (1ll << 40) && (n <= 1 || *ld <= (1ll << 50) / n);
}

bool misaligned(const void *p, int size) { return ((uintptr_t)p & (uintptr_t)(size - 1)) != 0; }

}   // namespace
