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
// Bound by reading the logits once (at 16 bits an exponential per element comes to three quarters of what the special function units
// give in that time).  One pass: every thread keeps the largest logit it met, the sums relative to it and where it was.  What
// follows touches little of the row again:
//   - the sum of the thread that met the largest logit of the block is taken once more without it (that thread's elements alone);
//   - the k-th largest of the threads' maxima bounds the k-th largest logit from below, so the alternatives lie with the few threads
//     whose maximum reaches it: their elements are read again, by all threads, and ranked by counting.
// Few rows: up to eight blocks of a cluster share a row and join their sums and alternatives through distributed shared memory.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "f8_real.cuh"

namespace {

constexpr int LP_THREADS = 256;
// Vectors of 16 bytes a thread takes at once, and blocks an SM has room for (64 registers a thread).  What overlaps loads with arithmetic
// here is other blocks: 1024 x 50001 float, entropy: 4 and 4 38 us; 8 and 3 42; 4, the next 4 ahead in registers, and 3 43; three
// stages of 4 through shared memory and 3 40; 2 and 6 51; 4 and 5 41.
constexpr int LP_UNROLL = 4;
constexpr int LP_BLOCKS = 4;
// Vectors that a thread of a block with a whole row keeps in registers where the row has no more, so that it is not read again for the
// owner's elements and the alternatives.  256 rows of 1000 codes, 5 alternatives: none kept 5.7 us, two 5.2, four 5.3; 1024 x 50001 float:
// none and two 38.3 us, four 39.8 (registers).  Clusters keep none: eight in 96 registers, two blocks an SM, took 17.7 us for 16 rows of
// 131072 bf16 and 20 alternatives against 12.5.
constexpr int LP_KEEP = 2;
constexpr int LP_CANDIDATES = 1024;       // rows with more (as when one thread's elements hold most of the large ones) take the slow way
constexpr int LP_MOST_TOP = 32;

struct LpParams {
    int v, tokens, top;
    float c, cl, back;                      // inverse temperature, the same times log2(e), and c / cl (of cl as it is, rounded)
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

typedef unsigned long long Key;             // order and index of a logit: the larger logit first, then the smaller index; 0: none
__device__ __forceinline__ Key make_key(uint32_t order, int index) { return (Key)order << 32 | (uint32_t)~index; }
__device__ __forceinline__ int key_index(Key k) { return (int)~(uint32_t)k; }

struct MaxOp { __device__ __forceinline__ Key operator()(Key a, Key b) const { return a > b ? a : b; } };

// What differs between real logits and codes: the largest value is a float or an integer, and so is the difference before it is rounded.
template <typename T> struct Num {
    typedef float V;
    static constexpr int VEC = 16 / sizeof(T);
    static __device__ __forceinline__ V lowest() { return -INFINITY; }
    static __device__ __forceinline__ uint32_t order(V v) { return order_of(v); }
    static __device__ __forceinline__ V value(uint32_t o) { return value_of(o); }
    static __device__ __forceinline__ V larger(V a, V b) { return fmaxf(a, b); }
    static __device__ __forceinline__ V safe(V m) { return m == -INFINITY ? 0.f : m; }      // a reference to subtract: -infinity - -infinity is NaN
    static __device__ __forceinline__ float minus(V x, V m) { return x - m; }
    static __device__ __forceinline__ F2 minus2(V x, V y, V m) { return add2(pair(x, y), both(-m)); }
    static __device__ __forceinline__ V one(const T *p) { return to_float(*p); }
    static __device__ __forceinline__ void unpack(const uint4 &w, V (&x)[VEC]) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) {
                x[i] = __uint_as_float(u[i]);
            } else if constexpr (std::is_same<T, __half>::value) {
                const float2 f = __half22float2(*(const __half2 *)&u[i]);
                x[2 * i] = f.x;
                x[2 * i + 1] = f.y;
            } else {
                x[2 * i] = __uint_as_float(u[i] << 16);
                x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
            }
        }
    }
    static __device__ __forceinline__ bool bad(uint32_t top) { return top >= 0xff800000u; }       // +infinity or NaN
    static __device__ __forceinline__ bool empty(uint32_t top) { return top == 0x007fffffu; }     // -infinity
};
template <> struct Num<int> {
    typedef int V;
    static constexpr int VEC = 4;
    static __device__ __forceinline__ V lowest() { return (int)0x80000000; }
    static __device__ __forceinline__ uint32_t order(V v) { return (uint32_t)v ^ 0x80000000u; }
    static __device__ __forceinline__ V value(uint32_t o) { return (int)(o ^ 0x80000000u); }
    static __device__ __forceinline__ V larger(V a, V b) { return max(a, b); }
    static __device__ __forceinline__ V safe(V m) { return m; }
    static __device__ __forceinline__ float minus(V x, V m) { return -(float)((uint32_t)m - (uint32_t)x); }       // m >= x
    static __device__ __forceinline__ F2 minus2(V x, V y, V m) { return pair(minus(x, m), minus(y, m)); }
    static __device__ __forceinline__ V one(const int *p) { return *p; }
    static __device__ __forceinline__ void unpack(const uint4 &w, V (&x)[4]) { x[0] = (int)w.x; x[1] = (int)w.y; x[2] = (int)w.z; x[3] = (int)w.w; }
    static __device__ __forceinline__ bool bad(uint32_t) { return false; }
    static __device__ __forceinline__ bool empty(uint32_t) { return false; }
};

// Sums over some of the elements x relative to m: with z = (x - m) c log2(e), s of 2^z and t of z 2^z, each in two halves.  (t in z and not in
// x - m: of that the sum over a row passes the largest float where c is small and the logits are as large.)
template <typename T>
struct Sums {
    typedef typename Num<T>::V V;
    V m;
    F2 s, t;
    // two more elements, at most m
    __device__ __forceinline__ void add(V x, V y, V ref, float cl) {
        const float2 z = halves(mul2(Num<T>::minus2(x, y, ref), both(cl)));
        const F2 e = pair(exp2_fast(z.x), exp2_fast(z.y));
        s = add2(s, e);
        t = fma2(e, pair(fmaxf(z.x, -3e38f), fmaxf(z.y, -3e38f)), t);       // (0 * infinity)
    }
    __device__ __forceinline__ void add(V x, V ref, float cl) {
        const float z = Num<T>::minus(x, ref) * cl, e = exp2_fast(z);
        s = add2(s, pair(e, 0.f));
        t = fma2(pair(e, 0.f), pair(fmaxf(z, -3e38f), 0.f), t);
    }
    // the sums relative to a larger m (which is none of the elements met so far).  f z first, which is small wherever f is: s z of a mask of
    // low numbers is -infinity, and 0 times that NaN.
    __device__ __forceinline__ void raise(V to, float cl) {
        const float z = fmaxf(Num<T>::minus(m, to) * cl, -3e38f), f = exp2_fast(z);
        t = fma2(s, both(f * z), mul2(both(f), t));
        s = mul2(s, both(f));
        m = to;
    }
    __device__ __forceinline__ float sum_s() const { const float2 f = halves(s); return f.x + f.y; }
    __device__ __forceinline__ float sum_t() const { const float2 f = halves(t); return f.x + f.y; }
};

// What a block has found of its part of the row: read by the leading block of the cluster.
struct LpPart {
    Key best;                               // 0: the part has no element
    float r, t;                             // sums without the best element, relative to it
    int too_many;                           // more candidates than there is room for
    Key top[LP_MOST_TOP];                   // the part's alternatives in falling order, 0 behind the last
};

// how many of n keys are larger
__device__ __forceinline__ int above_in(const Key *keys, int n, Key k) {
    int above = 0, j = 0;
    for (; j + 8 <= n; j += 8) {
#pragma unroll
        for (int u = 0; u < 8; ++u) above += keys[j + u] > k ? 1 : 0;
    }
    for (; j < n; ++j) above += keys[j] > k ? 1 : 0;
    return above;
}

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_block(const void *p, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ Key remote64(uint32_t a) { Key v; asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory"); return v; }
__device__ __forceinline__ uint32_t remote32(uint32_t a) { uint32_t v; asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory"); return v; }

// KEEP: see LP_KEEP.
template <typename T, bool CLUSTER, int KEEP>
__global__ void __launch_bounds__(LP_THREADS, LP_BLOCKS) logprobs_kernel(LpParams p) {
    wait_for_stream();
    let_stream_go_on();
    typedef Num<T> N;
    typedef typename N::V V;
    constexpr int VEC = N::VEC;
    __shared__ Key room[2][32];
    __shared__ float froom[2][32];
    __shared__ Key keys[LP_MOST_TOP], found[LP_CANDIDATES];          // the row's alternatives; what they are taken from
    __shared__ int members[LP_THREADS];
    __shared__ int counts[4];               // candidates; threads to read again; the owner of the largest element; threads worth a look
    __shared__ LpPart part;
    const int tid = threadIdx.x;
    const long long row = CLUSTER ? blockIdx.y : blockIdx.x;
    const uint32_t rank = CLUSTER ? cluster_rank() : 0u, ranks = CLUSTER ? gridDim.x : 1u;
    const T *l = (const T *)p.logits + row * p.ldl;
    const float cl = p.cl;
    // the row: `head` elements in front of the first multiple of 16 bytes, whole vectors, `tail` elements; this block's part of them
    const int off = (int)((uintptr_t)l / sizeof(T) % VEC);
    const int head_all = off ? min(VEC - off, p.v) : 0, vecs_all = (p.v - head_all) / VEC;
    const int each = (vecs_all + (int)ranks - 1) / (int)ranks, v0 = min((int)rank * each, vecs_all), vecs = min(each, vecs_all - v0);
    const int first = head_all + v0 * VEC;                 // element at which the part's vectors start
    const int head = rank == 0 ? head_all : 0, tail = rank == ranks - 1 ? p.v - head_all - vecs_all * VEC : 0;
    const int tail_at = head_all + vecs_all * VEC;
    if (tid < 4) counts[tid] = 0;

    // ---- one pass: a thread takes every 256th vector, the first threads an element of the head or the tail
    Sums<T> sum;
    sum.m = N::lowest();
    sum.s = sum.t = 0ull;
    bool some = false;
    int at = 0, span = 0;                   // where the largest element lies: at .. at + span
    auto meet = [&](V x, int index) {
        if (!some || x > sum.m) {
            if (some) sum.raise(x, cl);
            sum.m = x;
            at = index;
            span = 0;
            some = true;
        }
        sum.add(x, N::safe(sum.m), cl);
    };
    // an element of the head or the tail
    const int edge_at = tid < head ? tid : tid >= 32 && tid - 32 < tail ? tail_at + tid - 32 : -1;
    const V edge = edge_at >= 0 ? N::one(l + edge_at) : N::lowest();
    if (tid < head) meet(edge, edge_at);
    const T *vl = l + first;
    auto batch = [&](const uint4 *w, int count, int base) {
        V x[LP_UNROLL][VEC];
        V top = N::lowest();
        int which = 0;
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u) {
            if (u >= count) break;
            N::unpack(w[u], x[u]);
            V most = x[u][0];
#pragma unroll
            for (int k = 1; k < VEC; ++k) most = N::larger(most, x[u][k]);
            if (u == 0 || most > top) { top = most; which = u; }
        }
        if (!some || top > sum.m) {
            if (some) sum.raise(top, cl);
            sum.m = top;
            at = first + (base + which * LP_THREADS) * VEC;
            span = VEC - 1;
            some = true;
        }
        const V ref = N::safe(sum.m);
#pragma unroll
        for (int u = 0; u < LP_UNROLL; ++u) {
            if (u >= count) break;
#pragma unroll
            for (int k = 0; k < VEC; k += 2) sum.add(x[u][k], x[u][k + 1], ref, cl);
        }
    };
    auto vector = [&](int i) {
        uint4 w;
        asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "l"(vl + (long long)i * VEC) : "memory");
        return w;
    };
    const int rounds = (vecs + LP_THREADS - 1) / LP_THREADS;
    const bool resident = KEEP && rounds <= KEEP;
    uint4 w[KEEP ? KEEP : 1];
    if (resident) {
#pragma unroll
        for (int u = 0; u < KEEP; ++u) w[u] = tid + u * LP_THREADS < vecs ? vector(tid + u * LP_THREADS) : make_uint4(0, 0, 0, 0);
        V top = N::lowest();
        int which = -1;
#pragma unroll
        for (int u = 0; u < KEEP; ++u) {
            if (tid + u * LP_THREADS >= vecs) continue;
            V x[VEC];
            N::unpack(w[u], x);
            V most = x[0];
#pragma unroll
            for (int k = 1; k < VEC; ++k) most = N::larger(most, x[k]);
            if (which < 0 || most > top) { top = most; which = u; }
        }
        if (which >= 0 && (!some || top > sum.m)) {
            if (some) sum.raise(top, cl);
            sum.m = top;
            at = first + (tid + which * LP_THREADS) * VEC;
            span = VEC - 1;
            some = true;
        }
        const V ref = N::safe(sum.m);
#pragma unroll
        for (int u = 0; u < KEEP; ++u) {
            if (tid + u * LP_THREADS >= vecs) continue;
            V x[VEC];
            N::unpack(w[u], x);
#pragma unroll
            for (int k = 0; k < VEC; k += 2) sum.add(x[k], x[k + 1], ref, cl);
        }
    } else {
        int i = tid;
        uint4 v[LP_UNROLL];
        for (; i + (LP_UNROLL - 1) * LP_THREADS < vecs; i += LP_UNROLL * LP_THREADS) {
#pragma unroll
            for (int u = 0; u < LP_UNROLL; ++u) v[u] = vector(i + u * LP_THREADS);
            batch(v, LP_UNROLL, i);
        }
        for (; i < vecs; i += LP_THREADS) {
            v[0] = vector(i);
            batch(v, 1, i);
        }
    }
    if (edge_at >= tail_at) meet(edge, edge_at);

    // ---- the block's largest element and the sums without it
    const uint32_t mine = N::order(sum.m);
    const Key high = some ? make_key(mine, at) : 0, low = some ? make_key(mine, at + span) : 0;      // bounds of the key of this thread's largest
    Key best = block_reduce<LP_THREADS>(high, MaxOp(), room[0]);
    V m = N::value((uint32_t)(best >> 32));
    bool lost = Num<T>::empty((uint32_t)(best >> 32));       // nothing but -infinity so far (or NaN, which the sums show)
    const bool owner = some && high == best;
    if (owner) counts[2] = tid;
    {
        float s = 0.f, t = 0.f;
        if (some) {
            const float z = lost ? 0.f : fmaxf(N::minus(sum.m, m) * cl, -3e38f), f = exp2_fast(z);
            const float own_s = sum.sum_s(), own_t = sum.sum_t();
            t = fmaf(own_s, f * z, f * own_t);              // (see raise)
            s = owner ? 0.f : f * own_s;
            if (owner && own_s != own_s) s = own_s;
        }
        __syncthreads();
        // the owner's elements once more, by all threads: exp of all but the first that equals the largest
        const int who = counts[2];
        bool seen = false;
        Key exact = 0;
        const int own_at = key_index(best);
        auto again = [&](V x, int index, bool here) {
            if (here && !seen && x == m) { seen = true; exact = make_key(N::order(x), index); return; }
            if (!lost) s += exp2_fast(N::minus(x, m) * cl);
        };
        if (best) {
            if (resident) {
                if (tid == who) {
#pragma unroll
                    for (int u = 0; u < KEEP; ++u) {
                        if (tid + u * LP_THREADS >= vecs) continue;
                        V x[VEC];
                        N::unpack(w[u], x);
                        const int index = first + (tid + u * LP_THREADS) * VEC;
#pragma unroll
                        for (int k = 0; k < VEC; ++k) again(x[k], index + k, index == own_at);
                    }
                }
            } else {
                for (int j = tid; j * LP_THREADS + who < vecs; j += LP_THREADS) {
                    V x[VEC];
                    N::unpack(vector(j * LP_THREADS + who), x);
                    const int index = first + (j * LP_THREADS + who) * VEC;
#pragma unroll
                    for (int k = 0; k < VEC; ++k) again(x[k], index + k, index == own_at);
                }
            }
            if (tid == who && edge_at >= 0) again(edge, edge_at, edge_at == own_at);
        }
        s = block_reduce<LP_THREADS>(s, SumOp(), froom[0]);
        t = block_reduce<LP_THREADS>(t, SumOp(), froom[1]);
        best = block_reduce<LP_THREADS>(exact, MaxOp(), room[1]);       // with its own index now
        if (tid == 0) {
            part.best = best;
            part.r = s;
            part.t = t;
            part.too_many = 0;
        }
    }

    // ---- the part's alternatives
    if (p.top == 1) {
        if (tid == 0) part.top[0] = best;
    } else if (p.top > 1) {
        // maxima of groups of eight threads; the top-th largest of the 32 bounds the threads worth a look ...
        Key g = low;
#pragma unroll
        for (int d = 4; d > 0; d >>= 1) g = max(g, __shfl_xor_sync(0xffffffffu, g, d));
        if ((tid & 7) == 0) room[0][tid >> 3] = g;
        __syncthreads();
        g = room[0][tid & 31];
        int above = 0;
#pragma unroll
        for (int j = 0; j < 32; ++j) above += room[0][j] > g ? 1 : 0;
        Key bound = above >= p.top - 1 ? g : 0;             // keys differ unless they are 0, so one lane has exactly top - 1 above it (or all the rest are 0)
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) bound = max(bound, __shfl_xor_sync(0xffffffffu, bound, d));
        // ... and the top-th largest of their own maxima is the bound of the elements
        Key least = bound;
        // (a thread with a handful of vectors is read again sooner than its worth is looked into; but a short row has fewer groups than
        // alternatives, no bound, and would rank all its elements: 2048 rows of 1000 bf16, top 20, 30 us so and 319 us)
        if (rounds > 4 || !bound) {
            // (counted in a counter of their own: one that is set to zero again between two uses needs a barrier on either side of that)
            if (low >= bound && low) found[atomicAdd(&counts[3], 1)] = low;
            __syncthreads();
            const int threads = counts[3];
            if (tid < threads && above_in(found, threads, found[tid]) == p.top - 1) room[1][0] = found[tid];
            __syncthreads();                                // (and the candidates below may go where the maxima were)
            least = threads >= p.top ? room[1][0] : 0;      // (fewer threads with elements than alternatives: all elements)
        }
        auto offer = [&](V x, int index) {
            const Key k = make_key(N::order(x), index);
            if (k < least) return;
            const int n = atomicAdd(&counts[0], 1);
            if (n < LP_CANDIDATES) found[n] = k;
        };
        if (resident) {
            if (some && high >= least) {
#pragma unroll
                for (int u = 0; u < KEEP; ++u) {
                    if (tid + u * LP_THREADS >= vecs) continue;
                    V x[VEC];
                    N::unpack(w[u], x);
                    V most = x[0];
#pragma unroll
                    for (int k = 1; k < VEC; ++k) most = N::larger(most, x[k]);
                    const int index = first + (tid + u * LP_THREADS) * VEC;
                    if (make_key(N::order(most), index) < least) continue;
#pragma unroll
                    for (int k = 0; k < VEC; ++k) offer(x[k], index + k);
                }
            }
        } else {
            if (some && high >= least) members[atomicAdd(&counts[1], 1)] = tid;
            __syncthreads();
            const int who = counts[1];
            for (int j = tid; j < who * rounds; j += LP_THREADS) {
                const int at_vec = (j / who) * LP_THREADS + members[j % who];
                if (at_vec >= vecs) continue;
                V x[VEC];
                N::unpack(vector(at_vec), x);
#pragma unroll
                for (int k = 0; k < VEC; ++k) offer(x[k], first + at_vec * VEC + k);
            }
        }
        if (edge_at >= 0) offer(edge, edge_at);
        if (tid < LP_MOST_TOP) part.top[tid] = 0;
        __syncthreads();
        const int n = counts[0];
        if (n > LP_CANDIDATES) {
            if (tid == 0) part.too_many = 1;
        } else {
            for (int j = tid; j < n; j += LP_THREADS) {
                const int n_above = above_in(found, n, found[j]);
                if (n_above < p.top) part.top[n_above] = found[j];
            }
        }
    }
    __syncthreads();

    // ---- the leading block joins the parts
    if (CLUSTER) cluster_sync();
    if (rank == 0) {
        float r = part.r, t = part.t;
        bool slow = part.too_many != 0;
        if (CLUSTER) {
            Key top = 0;
            for (uint32_t b = 0; b < ranks; ++b) top = max(top, remote64(in_block(&part.best, b)));
            m = N::value((uint32_t)(top >> 32));
            lost = Num<T>::empty((uint32_t)(top >> 32));
            r = t = 0.f;
            for (uint32_t b = 0; b < ranks; ++b) {
                const Key k = remote64(in_block(&part.best, b));
                const float br = __uint_as_float(remote32(in_block(&part.r, b))), bt = __uint_as_float(remote32(in_block(&part.t, b)));
                slow = slow || remote32(in_block(&part.too_many, b));
                if (!k && br == br) continue;               // no element (or nothing but NaN)
                if (k == top) {
                    r += br;
                    t += bt;
                } else {
                    const float z = lost ? 0.f : fmaxf(N::minus(N::value((uint32_t)(k >> 32)), m) * cl, -3e38f), f = exp2_fast(z);
                    r += f * (1.f + br);
                    t += fmaf(1.f + br, f * z, f * bt);
                }
            }
            best = top;
            // alternatives of all parts, ranked by counting
            if (p.top > 0) {
                const int per = p.top, all = per * (int)ranks;
                for (int j = tid; j < all; j += LP_THREADS) found[j] = remote64(in_block(&part.top[j % per], (uint32_t)(j / per)));
                __syncthreads();
                Key mine_top = 0;
                int n_above = LP_MOST_TOP;
                if (tid < all) {
                    mine_top = found[tid];
                    n_above = above_in(found, all, mine_top);
                }
                __syncthreads();
                if (mine_top && n_above < per) keys[n_above] = mine_top;
                __syncthreads();
            }
        } else {
            if (tid < p.top) keys[tid] = part.top[tid];
            __syncthreads();
        }
        const uint32_t top = (uint32_t)(best >> 32);
        const bool bad = r != r || t != t || !best || N::bad(top), empty = N::empty(top);
        const float nan = __int_as_float(0x7fffffff), lse = log1pf(r);
        auto logprob = [&](V x) { return bad ? nan : empty ? -INFINITY : N::minus(x, m) * p.c - lse; };
        if (tid == 0 && p.entropy) p.entropy[row] = bad ? nan : empty ? 0.f : lse - t * p.back / (1.f + r);
        if (p.lp)
            for (int j = tid; j < p.tokens; j += LP_THREADS) {
                const int64_t id = p.ids[row * p.tokens + j];
                p.lp[row * p.tokens + j] = id < 0 ? 0.f : id >= p.v ? nan : logprob(N::one(l + id));
            }
        if (!slow && !bad) {
            if (tid < p.top) {
                if (p.top_lp) p.top_lp[row * p.top + tid] = logprob(N::value((uint32_t)(keys[tid] >> 32)));
                if (p.top_ids) p.top_ids[row * p.top + tid] = key_index(keys[tid]);
            }
        } else {
            // one alternative after the other, a pass over the row for each
            Key below = ~0ull;
            for (int j = 0; j < p.top; ++j) {
                Key next = 0;
                for (int q = tid; q < p.v; q += LP_THREADS) {
                    const Key k = make_key(N::order(N::one(l + q)), q);
                    if (k < below) next = max(next, k);
                }
                below = block_reduce<LP_THREADS>(next, MaxOp(), room[j & 1]);
                if (tid == 0) {
                    if (p.top_lp) p.top_lp[row * p.top + j] = logprob(N::value((uint32_t)(below >> 32)));
                    if (p.top_ids) p.top_ids[row * p.top + j] = key_index(below);
                }
            }
        }
    }
    __syncwarp();                           // the barrier of the cluster takes all lanes together
    if (CLUSTER) cluster_sync();            // no block goes while the leader may read it
}

// Blocks that share a row: enough of them to give every SM about two, as long as each has 16 KiB of the row.  16 rows of 131072 bf16,
// 20 alternatives: one block a row 18.0 us, eight 12.6 us.
int lp_blocks(long long n, long long row_bytes) {
    int s = 1;
    while (s < 8 && n * s < 296 && row_bytes / (2 * s) >= 16384) s *= 2;
    return s;
}

template <typename T>
cudaError_t launch_logprobs(const LpParams &p, long long n, cudaStream_t st) {
    const int s = n <= 65535 ? lp_blocks(n, (long long)p.v * sizeof(T)) : 1;
    if (s == 1) return launch_early(logprobs_kernel<T, false, LP_KEEP>, dim3((unsigned)n), LP_THREADS, 0, st, p);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)s, (unsigned)n);
    cfg.blockDim = dim3(LP_THREADS);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)s;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, logprobs_kernel<T, true, 0>, p);
}

}   // namespace

extern "C" f8_status f8_token_logprobs(const f8_logprobs_desc *desc, const void *logits, const int64_t *tokens, float *logprobs, float *entropy,
                                       float *top_logprobs, int64_t *top_ids, void *cuda_stream) {
    if (!desc) return f8_set_error(F8_ERR_NULL, "descriptor is NULL");
    f8_logprobs_desc d = *desc;
    if (d.n < 0 || d.n > 0x7fffffffll || d.v <= 0 || d.v > MOST_EXTENT || d.tokens < 0 || d.tokens > MOST_EXTENT)
        return f8_set_error(F8_ERR_SHAPE, "n in 0 .. 2^31 - 1, v in 1 .. 2^31 - 256 and tokens in 0 .. 2^31 - 256 are needed");
    if (d.top < 0 || d.top > 32 || d.top > d.v) return f8_set_error(F8_ERR_SHAPE, "top must be in 0 .. 32 and at most v");
    if (!(d.inv_temperature > 0.f) || !isfinite(d.inv_temperature)) return f8_set_error(F8_ERR_SHAPE, "inv_temperature must be positive and finite");
    const int size = d.dtype == F8_S32 ? 4 : real_size(d.dtype);
    if (!size) return f8_set_error(F8_ERR_DTYPE, "dtype must be F8_S32, F8_F32, F8_F16 or F8_BF16");
    if (d.dtype == F8_S32 && (d.fl < -8 || d.fl > 32)) return f8_set_error(F8_ERR_FL_RANGE, "fl outside [-8, 32]");
    const float c = d.dtype == F8_S32 ? ldexpf(d.inv_temperature, -d.fl) : d.inv_temperature;
    if (!(c > 0.f) || !isfinite(1.5f * c)) return f8_set_error(F8_ERR_SHAPE, "inv_temperature * 2^-fl leaves the range of 32-bit floats");
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
    const float cl = c * 1.44269504f;
    LpParams p = {d.v, d.tokens, top_logprobs || top_ids ? d.top : 0, c, cl, (float)((double)c / cl), d.ldl, logits, tokens, logprobs, entropy, top_logprobs, top_ids};
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = d.dtype == F8_S32   ? launch_logprobs<int>(p, d.n, st)
                          : d.dtype == F8_F32 ? launch_logprobs<float>(p, d.n, st)
                          : d.dtype == F8_F16 ? launch_logprobs<__half>(p, d.n, st)
                                              : launch_logprobs<__nv_bfloat16>(p, d.n, st);
    if (e != cudaSuccess) return f8_set_error(F8_ERR_CUDA, cudaGetErrorString(e));
    return F8_OK;
}
