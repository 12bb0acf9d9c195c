// What lies between two blocks of a transformer, in one pass over its rows (f8_norm_quantize):
//
//     t = r + beta * g(gate) * post(x);   v = pre(t);   a = max |v|;  s = a / 127;  i = 127 / a;  q = floor(v * i + 1/2)
//
// Bound by memory traffic: x, r (and a gate per token) are read once, t, q and the values written once; what a row needs besides is two to
// five sums over it.  Rows of up to 16384 elements stay in registers, a warp to 32 warps a row, while the next row is on its way.  A
// block walks many rows, and up to 8192 elements each thread keeps the factors of its 8 elements (norm weights, the post norm's already
// multiplied by beta and a gate that all rows share).  With rows to spare it takes two at once, which share sums, barriers and
// the division of the scales; what bounds it then is memory, 33 instructions an element behind it.
// 4096 x 8192 bf16, norms on both sides, channel gate, all outputs: 55 us, 5.5 TB/s.  On the way there: 32 elements a thread and the weights
// read again for every row 73 us (half of them came from the second-level cache); 16 elements, several rows a block and the
// factors in shared memory 72; 8 elements, one row at a time 64; two rows with the options of the call tested for each 58.
// The deviation comes from rsqrtf (within 2^-22) and the mean from a product with 1 / c (two roundings): each thread of a row works both out, and
// with sqrtf and divisions, half a step closer, the same call takes 58.9 us against 54.7.
// Longer rows take a kernel that reads the row again for every sum, from the caches.
// One row at a time: codes alone of 4096 x 8192 bf16 (RMS norm 40.2 us with two rows) take 49.4 us with a gate per token, 66.2 with a layer norm and its
// bias, and 149 where the rows are 8191 wide.  Above 8192 elements the weights are read again for every row (2048 x 16384 bf16: 78.2 us); 32-bit rows of that
// length with a residual find no room for the next row in shared memory (2048 x 16384 float: 118 us); rows of any length, 2048 x 20000 bf16: 434 us.
#include "f8_rowdeal.cuh"

namespace {

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
__global__ void __launch_bounds__(ROW_THREADS) long_norm_kernel(NormParams p) {
    wait_for_stream();
    let_stream_go_on();
    __shared__ float room[4][32];
    __shared__ uint32_t uroom[32];
    const long long row = blockIdx.x;
    const T *x = (const T *)p.x + row * p.ldx, *g = p.gate ? (const T *)p.gate + row * p.ldg : nullptr;
    const T *r = p.res ? (const T *)p.res + row * p.ldr : nullptr;
    T *sum = p.sum ? (T *)p.sum + row * p.lds : nullptr, *y = p.y ? (T *)p.y + row * p.ldy : nullptr;
    int8_t *q = p.q ? p.q + row * p.ldq : nullptr;
    // mean and 1 / deviation of what `f` gives over the row (the deviation from the mean: a second pass)
    auto measure = [&](int kind, auto f, float &mean, float &rstd, float (*room)[32]) {
        mean = 0.f;
        rstd = 1.f;
        if (kind == F8_NORM_NONE) return;
        if (kind == F8_NORM_LAYER) {
            float s = 0.f;
            for (int i = threadIdx.x; i < p.c; i += ROW_THREADS) s += f(i);
            mean = block_reduce<ROW_THREADS>(s, SumOp(), room[0]) / (float)p.c;
        }
        float s = 0.f;
        for (int i = threadIdx.x; i < p.c; i += ROW_THREADS) {
            const float z = f(i) - mean;
            s += z * z;
        }
        rstd = 1.f / sqrtf(block_reduce<ROW_THREADS>(s, SumOp(), room[1]) / (float)p.c + p.eps);
    };
    Norm<W> post = {(const W *)p.post_w, (const W *)p.post_b, 0.f, 1.f, p.weight_offset, p.post_norm != F8_NORM_NONE};
    Norm<W> pre = {(const W *)p.pre_w, (const W *)p.pre_b, 0.f, 1.f, p.weight_offset, p.pre_norm != F8_NORM_NONE};
    measure(p.post_norm, [&](int i) { return to_float(x[i]); }, post.mean, post.rstd, room);
    auto total = [&](int i) {
        float z = post(to_float(x[i]), i);
        if (g) z *= gate_value(to_float(g[i]), p.gate_act);
        return fmaf(p.branch_scale, z, r ? to_float(r[i]) : 0.f);
    };
    measure(p.pre_norm, total, pre.mean, pre.rstd, room + 2);
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


// Sums over R rows (one or two) that the threads of a block hold, each thread a part of every row.  Every warp writes its part to its own
// word of `room`, which no other reduction uses within two barriers.  Two rows share the steps: half of a warp's lanes add up one row, half the
// other.
template <int THREADS, int R>
__device__ __forceinline__ void row_sums(float (&v)[R], float (*room)[32]) {
    constexpr int WARPS = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if constexpr (R == 1) {
        v[0] = warp_reduce(v[0], SumOp());
        if (THREADS == 32) return;
        if (lane == 0) room[0][warp] = v[0];
        __syncthreads();
        v[0] = room[0][lane & (WARPS - 1)];
#pragma unroll
        for (int d = WARPS / 2; d > 0; d >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], d);
    } else {
        const bool second = lane & 16;
        float w = (second ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, second ? v[0] : v[1], 16);
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) w += __shfl_xor_sync(0xffffffffu, w, d);
        if (THREADS != 32) {
            if ((lane & 15) == 0) room[second][warp] = w;
            __syncthreads();
            const float *const part = room[second];
            w = part[lane & (WARPS >= 16 ? 15 : WARPS - 1)];
            if (WARPS == 32) w += part[16 + (lane & 15)];
#pragma unroll
            for (int d = WARPS >= 16 ? 8 : WARPS / 2; d > 0; d >>= 1) w += __shfl_xor_sync(0xffffffffu, w, d);
        }
        v[0] = __shfl_sync(0xffffffffu, w, 0);
        v[1] = __shfl_sync(0xffffffffu, w, 16);
    }
}
// The largest of a magnitude each, in two halves with a barrier between them (that of the sums, where there are any): `wait` is the second.
template <int THREADS, int R>
__device__ __forceinline__ void row_peaks(uint32_t (&top)[R], uint32_t (*room)[32], bool wait) {
    constexpr int WARPS = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (!wait) {            // first half: before the barrier
            top[r] = warp_reduce(top[r], UMaxOp());
            if (THREADS != 32 && lane == 0) room[r][warp] = top[r];
        } else if (THREADS != 32) {
            top[r] = warp_reduce(room[r][lane & (WARPS - 1)], UMaxOp());
        }
    }
}

template <typename T, RowMode MODE, int THREADS, int E, int R>
__global__ void __launch_bounds__(row_block(THREADS), row_blocks(THREADS)) row_norm_kernel(NormParams p, bool w32, long long n) {
    wait_for_stream();
    let_stream_go_on();
    constexpr int BLOCK = row_block(THREADS), GROUPS = BLOCK / THREADS;
    extern __shared__ uint4 smem[];
    __shared__ float rooms[2][4][R][32];
    __shared__ uint32_t urooms[2][R][32];
    using D = Deal<T, MODE, THREADS, E>;
    constexpr int PER = D::PER, PAIRS = D::PAIRS;
    constexpr bool PIPE = MODE != LOOSE, KEEP = E == 8;       // (rows of a block lie alike: they meet the same weights)
    const float per = 1.f / (float)p.c;
    // Two rows at once only between blocks as most models have them, whose options the compiler then knows: a residual sum that is kept, no gate
    // per token, RMS norms without biases, codes.
    constexpr bool COMMON = R == 2;
    const bool own_gate = !COMMON && p.gate && p.ldg, fold = COMMON || !p.post_b, has_res = COMMON || p.res, has_sum = COMMON || p.sum, has_q = COMMON || p.q;
    const int post_norm = COMMON && p.post_norm != F8_NORM_NONE ? (int)F8_NORM_RMS : p.post_norm;
    const int tensors = 1 + (has_res ? 1 : 0) + (own_gate ? 1 : 0), gate_at = tensors - 1;
    const Ring<BLOCK, PER> ring(smem, R * tensors);
    // rows row, row + step, .. of a round of R; then R * step further
    const uint32_t step = gridDim.x * GROUPS, rows = (uint32_t)n;
    uint32_t row = GROUPS == 1 ? blockIdx.x : threadIdx.x / THREADS * gridDim.x + blockIdx.x;
    const uint32_t bx = (uint32_t)p.ldx * sizeof(T), br = (uint32_t)p.ldr * sizeof(T), bg = (uint32_t)p.ldg * sizeof(T);
    const uint32_t bs = (uint32_t)p.lds * sizeof(T), by = (uint32_t)p.ldy * sizeof(T), bq = (uint32_t)p.ldq;
    const D d(row_at((const T *)p.x, row, bx), p.c);
    auto send = [&](uint32_t first, int stage) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t at = first + r * step;
            if (at >= rows) continue;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                d.send(row_at((const T *)p.x, at, bx), j, ring.place(stage, r * tensors, j));
                if (has_res) d.send(row_at((const T *)p.res, at, br), j, ring.place(stage, r * tensors + 1, j));
                if (own_gate) d.send(row_at((const T *)p.gate, at, bg), j, ring.place(stage, r * tensors + gate_at, j));
            }
        }
        ring_commit();
    };
    if (PIPE) {
        ring.clear(d);
        send(row, 0);
    }
    auto weight = [&](const void *w, int i) { return w ? (sizeof(T) == 4 || w32 ? ((const float *)w)[i] : to_float(((const T *)w)[i])) + p.weight_offset : 1.f; };
    // the factor of x / deviation in the residual sum: weight, beta and a shared gate (with a bias behind the post norm the weight alone)
    auto post_weight = [&](int i) {
        float f = weight(p.post_w, i);
        if (!fold) return f;
        f *= p.branch_scale;
        return p.gate && !own_gate ? f * gate_value(to_float(((const T *)p.gate)[i]), p.gate_act) : f;
    };
    auto factor = [&](int j, F2 (&f)[PAIRS], bool post) {
        float e[D::VEC];
#pragma unroll
        for (int k = 0; k < D::VEC; ++k) {
            const int i = d.at(j, k);
            e[k] = !d.in(j, k) ? 0.f : post ? post_weight(i) : weight(p.pre_w, i);
        }
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) f[i] = pair(e[2 * i], e[2 * i + 1]);
    };
    F2 kept[KEEP ? 2 : 1][PER][PAIRS];
    if (KEEP) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            factor(j, kept[0][j], true);
            factor(j, kept[KEEP ? 1 : 0][j], false);
        }
    }
    auto activate_gate = [&](F2 (&f)[PAIRS]) {
        if (p.gate_act == F8_ACT_NONE) return;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            const float2 g = halves(f[i]);
            f[i] = pair(gate_value(g.x, p.gate_act), gate_value(g.y, p.gate_act));
        }
    };
    for (int stage = 0; row < rows; row += R * step, stage ^= 1) {
        float (*const room)[R][32] = rooms[stage];
        uint32_t (*const uroom)[32] = urooms[stage];
        if (PIPE) {
            send(row + R * step, stage ^ 1);
            ring_wait();
        }
        F2 v[R][PER][PAIRS];
#pragma unroll
        for (int r = 0; r < R; ++r)         // (a second row that is not there: what the ring held before, which nothing is written from)
#pragma unroll
            for (int j = 0; j < PER; ++j)
                unpack<T>(PIPE ? d.take(j, ring.place(stage, r * tensors, j)) : d.load(row_at((const T *)p.x, row, bx), j), v[r][j]);
        // v <- (v - mean) / deviation
        auto standardize = [&](int kind, float (*rm)[R][32]) {
            float s[R];
            if (kind == F8_NORM_LAYER) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    F2 t = 0ull;
#pragma unroll
                    for (int j = 0; j < PER; ++j)
#pragma unroll
                        for (int i = 0; i < PAIRS; ++i) t = add2(t, v[r][j][i]);
                    const float2 h = halves(t);
                    s[r] = h.x + h.y;
                }
                row_sums<THREADS, R>(s, rm[0]);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const F2 mean = both(-s[r] * per);
#pragma unroll
                    for (int j = 0; j < PER; ++j) {
#pragma unroll
                        for (int i = 0; i < PAIRS; ++i) v[r][j][i] = add2(v[r][j][i], mean);
                        d.mask(j, v[r][j]);
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                F2 t = 0ull;
#pragma unroll
                for (int j = 0; j < PER; ++j)
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) t = fma2(v[r][j][i], v[r][j][i], t);
                const float2 h = halves(t);
                s[r] = h.x + h.y;
            }
            row_sums<THREADS, R>(s, rm[1]);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const F2 rstd = both(rsqrtf(s[r] * per + p.eps));
#pragma unroll
                for (int j = 0; j < PER; ++j)
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) v[r][j][i] = mul2(v[r][j][i], rstd);
            }
        };
        auto by_factors = [&](bool post) {
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                F2 f[PAIRS];
                if (!KEEP) factor(j, f, post);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) v[r][j][i] = mul2(v[r][j][i], KEEP ? kept[KEEP && !post ? 1 : 0][j][i] : f[i]);
            }
        };
        auto plus = [&](const void *b) {
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                if (!d.on(j)) continue;
                F2 f[PAIRS];
                if (sizeof(T) == 4 || w32) d.template weights<true>(b, j, f);
                else d.template weights<sizeof(T) == 4>(b, j, f);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) v[r][j][i] = add2(v[r][j][i], f[i]);
            }
        };
        if (post_norm != F8_NORM_NONE) standardize(post_norm, room);
        if (!fold) {
            by_factors(true);
            plus(p.post_b);
            if (p.gate && !own_gate) {
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    if (!d.on(j)) continue;
                    F2 f[PAIRS];
                    d.template weights<sizeof(T) == 4>(p.gate, j, f);
                    activate_gate(f);
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int i = 0; i < PAIRS; ++i) v[r][j][i] = mul2(v[r][j][i], f[i]);
                }
            }
        }
        if (own_gate) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    F2 f[PAIRS];
                    unpack<T>(PIPE ? d.take(j, ring.place(stage, r * tensors + gate_at, j)) : d.load(row_at((const T *)p.gate, row, bg), j), f);
                    activate_gate(f);
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) v[r][j][i] = mul2(v[r][j][i], f[i]);
                }
        }
        // the residual sum
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            F2 f[PAIRS];
            if (fold && KEEP) {
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) f[i] = kept[0][j][i];
            } else if (fold) {
                factor(j, f, true);
            } else {
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) f[i] = both(p.branch_scale);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (has_res) {
                    F2 t[PAIRS];
                    unpack<T>(PIPE ? d.take(j, ring.place(stage, r * tensors + 1, j)) : d.load(row_at((const T *)p.res, row, br), j), t);
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) v[r][j][i] = fma2(v[r][j][i], f[i], t[i]);
                } else {
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) v[r][j][i] = mul2(v[r][j][i], f[i]);
                }
                if (has_sum && (r == 0 || row + r * step < rows)) d.store(row_at((T *)p.sum, row + r * step, bs), j, v[r][j]);
            }
        }
        if (!has_q && !p.y) continue;
        float peak[R];
        uint32_t top[R];
        auto peaks = [&]() {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                peak[r] = 0.f;
#pragma unroll
                for (int j = 0; j < PER; ++j)
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) peak[r] = peak_of(peak[r], v[r][j][i]);
                top[r] = magnitude(peak[r]);
            }
            row_peaks<THREADS, R>(top, uroom, false);
        };
        if (COMMON || (has_q && p.pre_norm == F8_NORM_RMS && !p.pre_b)) {
            // the sum of squares and max |t w| over one barrier: v = (t w) * rstd, and the product with one rstd keeps the order
            float s[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                F2 t = 0ull;
#pragma unroll
                for (int j = 0; j < PER; ++j)
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) t = fma2(v[r][j][i], v[r][j][i], t);
                const float2 h = halves(t);
                s[r] = h.x + h.y;
            }
            by_factors(false);
            peaks();
            row_sums<THREADS, R>(s, room[2]);
            row_peaks<THREADS, R>(top, uroom, true);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float rstd = rsqrtf(s[r] * per + p.eps);
                top[r] = magnitude(__uint_as_float(top[r]) * rstd);
                const F2 f = both(rstd);
#pragma unroll
                for (int j = 0; j < PER; ++j)
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) v[r][j][i] = mul2(v[r][j][i], f);
            }
        } else {
            if (p.pre_norm != F8_NORM_NONE) {
                standardize(p.pre_norm, room + 2);
                by_factors(false);
                if (p.pre_b) plus(p.pre_b);
            }
            if (!has_q) {
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int j = 0; j < PER; ++j)
                        if (r == 0 || row + r * step < rows) d.store(row_at((T *)p.y, row + r * step, by), j, v[r][j]);
                continue;
            }
            peaks();
            if (THREADS != 32) __syncthreads();
            row_peaks<THREADS, R>(top, uroom, true);
        }
        RowScale s[R];
        RowScale::of_warp(top, s);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t at = row + r * step;
            if (r > 0 && at >= rows) continue;
            if ((THREADS == 32 ? threadIdx.x & 31 : threadIdx.x) == 0) p.scale[at] = s[r].scale;
            emit<T>(d, v[r], s[r], top[r] < 0x7f800000u, row_at(p.q, at, bq), p.y ? row_at((T *)p.y, at, by) : nullptr);
        }
    }
}

template <typename T, RowMode MODE, int THREADS, int E>
cudaError_t launch_row_norm_at(const NormParams &p, bool w32, long long n, cudaStream_t st) {
    constexpr int PER = E * (int)sizeof(T) / 16;
    const int tensors = 1 + (p.res ? 1 : 0) + (p.gate && p.ldg ? 1 : 0);
    if constexpr (MODE == PLAIN && E == 8 && THREADS != 32) {
        // two rows at once where every block has several rounds of them: what a thread pays for a row beside its elements it then pays for two
        const bool common = p.res && p.sum && p.q && !(p.gate && p.ldg) && p.post_norm != F8_NORM_LAYER && !p.post_b && p.pre_norm == F8_NORM_RMS && !p.pre_b;
        if (common && n >= 8ll * 148 * (1024 / THREADS) && ring_bytes(THREADS, PER, 2 * tensors) <= RING_MOST)
            return launch_ring<row_norm_kernel<T, MODE, THREADS, E, 2>>(THREADS, PER, 2 * tensors, n, st, p, w32);
    }
    if (MODE != LOOSE && ring_bytes(THREADS, PER, tensors) <= RING_MOST)
        return launch_ring<row_norm_kernel<T, MODE, THREADS, E, 1>>(THREADS, PER, tensors, n, st, p, w32);
    return launch_ring<row_norm_kernel<T, LOOSE, THREADS, E, 1>>(THREADS, PER, 0, n, st, p, w32);
}
template <typename T, RowMode MODE>
cudaError_t launch_row_norm(const NormParams &p, bool w32, long long n, cudaStream_t st) {
    const int need = p.c + (MODE == SHIFT ? 16 / (int)sizeof(T) - 1 : 0);
    if (need <= 32 * 8) return launch_row_norm_at<T, MODE, 32, 8>(p, w32, n, st);
    if (need <= 128 * 8) return launch_row_norm_at<T, MODE, 128, 8>(p, w32, n, st);
    if (need <= 256 * 8) return launch_row_norm_at<T, MODE, 256, 8>(p, w32, n, st);
    if (need <= 512 * 8) return launch_row_norm_at<T, MODE, 512, 8>(p, w32, n, st);
    if (need <= 1024 * 8) return launch_row_norm_at<T, MODE, 1024, 8>(p, w32, n, st);
    return launch_row_norm_at<T, MODE, 1024, 16>(p, w32, n, st);
}

template <typename T>
cudaError_t launch_norm(const NormParams &p, long long n, bool w32, cudaStream_t st) {
    constexpr int VEC = 16 / sizeof(T);
    RowLayout l(n, sizeof(T), p.c);
    l.add(p.x, p.ldx, sizeof(T));
    l.add(p.res, p.ldr, sizeof(T));
    l.add(p.sum, p.lds, sizeof(T));
    l.add(p.y, p.ldy, sizeof(T));
    l.add(p.q, p.ldq, 1);
    if (p.gate && p.ldg) l.add(p.gate, p.ldg, sizeof(T));
    if (p.gate && !p.ldg) l.vector(p.gate);
    l.vector(p.post_w);
    l.vector(p.post_b);
    l.vector(p.pre_w);
    l.vector(p.pre_b);
    if (l.near) {
        if (l.same && !l.shift() && p.c <= ROW_MOST) return launch_row_norm<T, PLAIN>(p, w32, n, st);
        if (l.same && p.c + VEC - 1 <= ROW_MOST) return launch_row_norm<T, SHIFT>(p, w32, n, st);
        if (p.c <= ROW_MOST) return launch_row_norm<T, LOOSE>(p, w32, n, st);
    }
    const dim3 grid((unsigned)n);
    if (w32) return launch_early(long_norm_kernel<T, float>, grid, ROW_THREADS, 0, st, p);
    return launch_early(long_norm_kernel<T, T>, grid, ROW_THREADS, 0, st, p);
}

}   // namespace

extern "C" f8_status f8_norm_quantize(const f8_norm_desc *desc, const void *x, const void *gate, const void *residual, const void *post_w,
                           const void *post_b, const void *pre_w, const void *pre_b, void *residual_out, int8_t *q, float *scale,
                           void *y, void *cuda_stream) {
    if (!desc) return f8_set_error(F8_ERR_NULL, "descriptor is NULL");
    f8_norm_desc d = *desc;
    if (d.n < 0 || d.n > 0x7fffffffll || d.c <= 0 || d.c > MOST_EXTENT) return f8_set_error(F8_ERR_SHAPE, "n in 0 .. 2^31 - 1 and c in 1 .. 2^31 - 256 are needed");
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
