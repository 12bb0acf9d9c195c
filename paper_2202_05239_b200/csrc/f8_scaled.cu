// f8_linear_scaled, from two rows on with the fifth-generation tensor cores (tcgen05.mma kind::i8, int32 accumulators in tensor memory).
//
//     y[i, j] = round( fma((float)acc * sx[i], sw[j], b[j]) ),   acc = sum_k x[i, k] w[j, k]
//
// scaled_token_kernel: one row of x, on the CUDA cores (below).
//
// scaled_split_kernel: products whose weights are read once or a few times (decoding batches, narrow layers).  A tile is 128 rows of x
// (as many as there are) by BN rows of w, its K divided among up to eight blocks of a cluster, so that all SMs fetch weights however
// few tiles there are; each block keeps its whole share of the weights on its way through a ring of bulk tensor copies.  The
// partial sums meet in shared memory and every block of the cluster finishes a part of the tile (integer sums: the order changes nothing).
//
// scaled_pair_kernel: products bound by the tensor cores.  Persistent pairs of blocks on 256 x 256 tiles (cta_group::2: each block holds 128 rows
// of x and 128 of w), two accumulators so that a tile leaves while the next is multiplied, tiles walked in groups of eight rows of tiles.
// 8192 x 4096 x 8192: 176 us (169 on another card), 3.1 POPS of the 4.2 that instructions alone reach; under the power cap of a long run 204 us (197).
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>

#include "f8_real.cuh"
#include "f8_tc_ptx.cuh"

namespace {

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

__device__ __forceinline__ float load_real(const void *p, int dtype, long long i) {
    return dtype == F8_F32 ? ((const float *)p)[i] : dtype == F8_F16 ? to_float(((const __half *)p)[i]) : to_float(((const __nv_bfloat16 *)p)[i]);
}
__device__ __forceinline__ void store_real(void *p, int dtype, long long i, float v) {
    if (dtype == F8_F32) ((float *)p)[i] = v;
    else if (dtype == F8_F16) ((__half *)p)[i] = from_float<__half>(v);
    else ((__nv_bfloat16 *)p)[i] = from_float<__nv_bfloat16>(v);
}
__device__ __forceinline__ float scaled(int acc, float sx, float sw, float b) { return __fmaf_rn(__fmul_rn(__int2float_rn(acc), sx), sw, b); }

// Bytes sh .. sh + 15 of two neighbouring granules of 16 bytes: by words, then by bytes.
__device__ __forceinline__ uint4 shift_bytes(uint4 a, uint4 b, uint32_t sh) {
    if (sh & 8u) { a.x = a.z; a.y = a.w; a.z = b.x; a.w = b.y; b.x = b.z; b.y = b.w; }
    if (sh & 4u) { a.x = a.y; a.y = a.z; a.z = a.w; a.w = b.x; b.x = b.y; }
    const uint32_t bits = (sh & 3u) * 8u;
    return make_uint4(__funnelshift_r(a.x, a.y, bits), __funnelshift_r(a.y, a.z, bits), __funnelshift_r(a.z, a.w, bits), __funnelshift_r(a.w, b.x, bits));
}
// The first n bytes, zeros behind them.
__device__ __forceinline__ uint4 first_bytes(uint4 v, int n) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int m = n - 4 * j;
        w[j] = m >= 4 ? w[j] : m <= 0 ? 0u : w[j] & (0xffffffffu >> (32 - 8 * m));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

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

constexpr int SC_KB = 128;                     // bytes of K in a chunk: one span of the swizzle
constexpr int SC_MAX_STAGES = 24;
constexpr int SC_CONTROL = 1024;
constexpr int SC_SMEM = 227 * 1024 - 1024;     // what a block may ask for, less the alignment of the ring

// In the first KiB of the aligned buffer, the barriers first, as in the other kernels: a late arrival meets a barrier.
struct ScControl {
    uint64_t full[SC_MAX_STAGES], empty[SC_MAX_STAGES];
    uint64_t tfull[2], tempty[2];
    uint32_t tmem;
    int abort_flag;
};

__device__ __forceinline__ uint32_t cluster_address(uint32_t a, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    return r;
}
__device__ __forceinline__ uint4 cluster_load(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}

// ----------------------------------------------------------------------------- K divided among the blocks of a cluster

struct SplitParams {
    ScaledParams s;
    int m_tiles, chunks, split, stages, a_rows;      // a_rows: rows of x a copy brings, a multiple of 8
    int soft_warps, slots;         // without bulk copies: warps that fetch, chunks on their way (4 or 8)
    uint32_t idesc;
    uint64_t desc;
    bool wide;
    int *status;
    unsigned long long wait_limit;
};

// Producer, issuer, four warps that read the accumulator; where bulk copies cannot fetch the operands (rows that do not start at multiples of
// 16 bytes: an odd K, a slice), up to sixteen more warps do: the granules of 16 bytes that hold a row's chunk come through raw slots in shared
// memory, are shifted together and written where the swizzle would put them.
constexpr int SPLIT_THREADS = 192, SOFT_THREADS = 512;
constexpr uint32_t SOFT_RAW = 16 * 144;       // bytes of a warp's slot: sixteen rows, nine granules each

template <int BN, bool SOFT>
__global__ void __launch_bounds__(SPLIT_THREADS + (SOFT ? SOFT_THREADS : 0), 1) scaled_split_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                                                                        const SplitParams p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t *const base = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    ScControl &ctl = *(ScControl *)base;
    float *const sw = (float *)(base + SC_CONTROL), *const bias = sw + BN, *const sx = bias + BN;     // of this tile
    uint8_t *const ring = base + 2 * SC_CONTROL + 1024;
    const uint32_t a_bytes = (uint32_t)p.a_rows * SC_KB, stage_bytes = a_bytes + BN * SC_KB;
    const uint32_t raw_at = smem_u32(ring), ring_at = raw_at + (SOFT ? ((uint32_t)(p.slots * p.soft_warps) * SOFT_RAW + 1023u) & ~1023u : 0u);
    const uint32_t full = smem_u32(&ctl.full[0]), empty = smem_u32(&ctl.empty[0]), tfull = smem_u32(&ctl.tfull[0]);
    const int warp = uniform((int)(threadIdx.x >> 5)), lane = threadIdx.x & 31;
    const int tile = (int)blockIdx.x / p.split, rank = (int)blockIdx.x % p.split;
    const int n_t = tile / p.m_tiles, m0 = (tile - n_t * p.m_tiles) * 128, n0 = n_t * BN;
    const int c0 = (int)((long long)p.chunks * rank / p.split), uses = (int)((long long)p.chunks * (rank + 1) / p.split) - c0;
    const WaitCtx wc = make_wait_ctx(&ctl.abort_flag, p.status, p.wait_limit);

    if (threadIdx.x == 0) {
        ctl.abort_flag = 0;
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full + 8 * s, SOFT ? p.soft_warps : 1);
            mbar_init(empty + 8 * s, 1);
        }
        mbar_init(tfull, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        if (!SOFT) prefetch_tensormap(&map_x);
        if (!SOFT) prefetch_tensormap(&map_w);
    }
    if (warp == 1) tmem_alloc(smem_u32(&ctl.tmem), BN);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(ctl.tmem);
    grid_dependency_wait();                    // the weights may come from earlier work in the stream as well
    grid_launch_dependents();

    if (SOFT && warp >= SPLIT_THREADS / 32) {
        // sixteen rows of the stage a warp: each chunk's nine granules of a row (one more than a chunk, for the shift) go to a raw slot of the
        // warp's own, as many chunks ahead as there are slots; then eight lanes a row shift and write them.
        const int pw = warp - SPLIT_THREADS / 32;
        if (pw < p.soft_warps) {
            const int all = p.a_rows + BN, r0 = 16 * pw;
            auto row_of = [&](int r) -> const uint8_t * {           // a row of the stage, null where the matrices have none
                r += r0;
                if (r < p.a_rows) return m0 + r < p.s.n ? p.s.x + (long long)(m0 + r) * p.s.ldx : nullptr;
                r -= p.a_rows;
                return r < BN && n0 + r < p.s.out ? p.s.w + (long long)(n0 + r) * p.s.ldw : nullptr;
            };
            const int j = lane & 7, q0 = lane >> 3;
            const uint8_t *src[5];                                  // granule j of rows q0, q0 + 4, .. ; the ninth granule of row `lane`
            uint32_t sh = 0;                                        // a byte each: the rows' distance from a multiple of 16
            int from[5];                                            // byte of the row at which the granule starts, in chunk 0 of this block
#pragma unroll
            for (int q = 0; q < 5; ++q) {
                const uint8_t *const row = row_of(q < 4 ? q0 + 4 * q : lane & 15);
                const uint32_t d = (uint32_t)(uintptr_t)row & 15u;
                if (q < 4) sh |= d << (8 * q);
                from[q] = c0 * SC_KB + (q < 4 ? 16 * j : 128) - (int)d;
                src[q] = row + from[q];
                // nothing to fetch: beyond every chunk
                if (!row || (q == 4 && (lane >= 16 || d == 0))) {
                    src[q] = p.s.w;
                    from[q] = 0x7fffffff - SC_KB * 4096;
                }
            }
            const uint32_t raw = raw_at + (uint32_t)pw * SOFT_RAW, slot_bytes = (uint32_t)p.soft_warps * SOFT_RAW;
            const uint32_t ninth = raw + (uint32_t)(lane & 15) * 144u + 128u, mine = raw + (uint32_t)q0 * 144u + 16u * j;
            auto fetch = [&](int u, int slot) {
                if (u < uses) {
#pragma unroll
                    for (int q = 0; q < 5; ++q) {
                        if (q == 4 && lane >= 16) break;
                        const bool some = from[q] + u * SC_KB < p.s.k;
                        const uint8_t *const g = some ? src[q] + (long long)u * SC_KB : (const uint8_t *)((uintptr_t)p.s.w & ~(uintptr_t)15);
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((q < 4 ? mine + 576u * q : ninth) + (uint32_t)slot * slot_bytes), "l"(g),
                                     "r"(some ? 16 : 0)
                                     : "memory");
                    }
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            for (int u = 0; u < p.slots - 1; ++u) fetch(u, u);
            int stage = 0, slot = 0;
            uint32_t phase = 0;
            for (int u = 0; u < uses; ++u) {
                fetch(u + p.slots - 1, slot == 0 ? p.slots - 1 : slot - 1);
                if (p.slots == 8) asm volatile("cp.async.wait_group 7;" ::: "memory");
                else asm volatile("cp.async.wait_group 3;" ::: "memory");
                __syncwarp();
                if (u >= p.stages && !warp_wait(empty + 8 * stage, phase ^ 1, wc, 153)) break;
                const uint32_t dst = ring_at + (uint32_t)stage * stage_bytes + (uint32_t)r0 * SC_KB;       // (rows of x, then of w: one behind the other)
                const int left = p.s.k - (c0 + u) * SC_KB - 16 * j;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int r = q0 + 4 * q;
                    const uint32_t at = mine + 576u * q + (uint32_t)slot * slot_bytes;
                    uint4 v = shift_bytes(lds128(at), lds128(at + 16), (sh >> (8 * q)) & 15u);
                    if (left < 16) v = first_bytes(v, left);
                    if (r0 + r < all) sts128(dst + (uint32_t)r * SC_KB + (((uint32_t)j ^ ((uint32_t)r & 7u)) << 4), v);
                }
                __syncwarp();                   // the slot is read: it may be filled again
                if (lane == 0) mbar_arrive(full + 8 * stage);
                if (++stage == p.stages) { stage = 0; phase ^= 1; }
                if (++slot == p.slots) slot = 0;
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        }
    } else if (SOFT && warp == 0) {
    } else if (warp == 0) {
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int u = 0; u < uses; ++u) {
            if (u >= p.stages && !warp_wait(empty + 8 * stage, phase ^ 1, wc, 150)) { ok = false; break; }
            const uint32_t dst = ring_at + (uint32_t)stage * stage_bytes, fb = full + 8 * stage;
            warp_expect_tx(fb, stage_bytes);
            tma_load_2d(dst + a_bytes, &map_w, fb, (c0 + u) * SC_KB, n0, lane == 0);
            tma_load_2d(dst, &map_x, fb, (c0 + u) * SC_KB, m0, lane == 0);
            if (++stage == p.stages) { stage = 0; phase ^= 1; }
        }
        if (!ok) {
            // the copies in flight must land before this block's shared memory may go: those of the last stage filled, or some time
            const unsigned long long t0 = clock64();
            while ((unsigned long long)(clock64() - t0) < 4000000ull) {
            }
        }
    } else if (warp == 1) {
        int stage = 0;
        uint32_t phase = 0;
        const uint32_t desc_hi = (uint32_t)(p.desc >> 32);
        for (int u = 0; u < uses; ++u) {
            if (!warp_wait(full + 8 * stage, phase, wc, 151)) break;
            // what the warps wrote, for the tensor cores to read (the fence stands here, behind the barrier: in the writers it would wait for
            // the loads they have on their way)
            if (SOFT) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            tc_fence_after();
            const uint32_t lo = (uint32_t)p.desc | (((ring_at + (uint32_t)stage * stage_bytes) & 0x3ffffu) >> 4);
            mma_i8_sub<4>(tmem, lo, lo + (a_bytes >> 4), desc_hi, p.idesc, u != 0 ? 1u : 0u);
            if (u + p.stages < uses) mma_commit(empty + 8 * stage);      // (no arrival that nobody waits for: it could meet the next block's barrier)
            if (++stage == p.stages) { stage = 0; phase ^= 1; }
        }
        mma_commit(tfull);
        const unsigned long long t0 = clock64();
        while (!mbar_try_wait(tfull, 0) && (unsigned long long)(clock64() - t0) < DRAIN_LIMIT_CYCLES) {
        }
        __syncwarp();
    } else {
        const int t = (int)threadIdx.x - 64;      // 0 .. 127
        for (int i = t; i < BN; i += 128) {
            const int o = n0 + i;
            sw[i] = o < p.s.out ? p.s.ws[p.s.w_scales == 1 ? 0 : o] : 0.f;
            bias[i] = p.s.bias && o < p.s.out ? load_real(p.s.bias, p.s.bias_dtype, o) : 0.f;
        }
        sx[t] = m0 + t < p.s.n ? p.s.xs[p.s.x_scales == 1 ? 0 : m0 + t] : 0.f;
    }
    // the accumulator is complete: the ring is free, and takes the partial sums
    if (warp >= 2 && warp < 6) {
        warp_wait(tfull, 0, wc, 152);
        tc_fence_after();
        const int rows = min(128, p.s.n - m0), row = 32 * (warp & 3) + lane;
        if (32 * (warp & 3) < rows) {
#pragma unroll
            for (int c = 0; c < BN; c += 16) {
                int v[16];
                tmem_ld16(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + c, v);
                tmem_ld_wait16(v);
                if (row < rows) {
                    const uint32_t at = ring_at + (uint32_t)(row * (BN + 4) + c) * 4;
#pragma unroll
                    for (int q = 0; q < 4; ++q) sts128(at + 16 * q, make_uint4((uint32_t)v[4 * q], (uint32_t)v[4 * q + 1], (uint32_t)v[4 * q + 2], (uint32_t)v[4 * q + 3]));
                }
                __syncwarp();                   // the next load takes all lanes together, also those without a row
            }
        }
        tc_fence_before();
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, BN);
    }
    if (p.split > 1) cluster_sync_all();
    {
        const int rows = min(128, p.s.n - m0), all = rows * (BN / 4);
        const int from = (int)((long long)all * rank / p.split), to = (int)((long long)all * (rank + 1) / p.split);
        for (int i = from + (int)threadIdx.x; i < to; i += (int)blockDim.x) {
            const int row = i / (BN / 4), c = (i - row * (BN / 4)) * 4, o = n0 + c;
            if (o >= p.s.out) continue;
            const uint32_t at = ring_at + (uint32_t)(row * (BN + 4) + c) * 4;
            int acc[4] = {0, 0, 0, 0};
            uint4 v[8];                         // all on their way before the first is added
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] = r < p.split ? cluster_load(cluster_address(at, (uint32_t)r)) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 8; ++r) { acc[0] += (int)v[r].x; acc[1] += (int)v[r].y; acc[2] += (int)v[r].z; acc[3] += (int)v[r].w; }
            const float w4[4] = {sw[c], sw[c + 1], sw[c + 2], sw[c + 3]}, b4[4] = {bias[c], bias[c + 1], bias[c + 2], bias[c + 3]};
            store_scaled4(p.s, acc, m0 + row, o, sx[row], w4, b4, p.wide && o + 4 <= p.s.out);
        }
    }
    __syncwarp();
    if (p.split > 1) cluster_sync_all();       // no block goes while another may read it
}

// ----------------------------------------------------------------------------- one row of x

// The product of one token is bound by reading the weights once and, up to some tens of megabytes, by the chain of one launch: here a row of
// w a warp, straight from memory into dot products of four bytes (dp4a), four loads of 16 bytes a lane on their way and as many of
// x out of the first-level cache, one integer reduction over the warp.  No shared memory, no barrier, nothing to set up.
// 4096 x 4096: 5.1 us (split kernel 6.7), 1024 x 8192: 3.6 (4.5), 8192 x 28672: 36.5, 6.4 TB/s (38.6).  Two rows a warp 5.6 / 3.1 / 37.6, eight
// loads 7.5 / 5.2 / 39.7; two tokens in this form 8.2 at 4096 x 4096 (split kernel 6.8).
constexpr int TOKEN_THREADS = 128, TOKEN_UNROLL = 4;

template <bool SIGNED>
__device__ __forceinline__ int dot4(uint32_t x, uint32_t w, int acc) {
    int d;
    if (SIGNED) asm("dp4a.s32.s32 %0, %1, %2, %3;" : "=r"(d) : "r"(x), "r"(w), "r"(acc));
    else asm("dp4a.u32.s32 %0, %1, %2, %3;" : "=r"(d) : "r"(x), "r"(w), "r"(acc));
    return d;
}

template <bool SIGNED>
__global__ void __launch_bounds__(TOKEN_THREADS) scaled_token_kernel(ScaledParams p) {
    wait_for_stream();
    let_stream_go_on();
    const int lane = threadIdx.x & 31;
    const long long o = (long long)blockIdx.x * (TOKEN_THREADS / 32) + (threadIdx.x >> 5);
    if (o >= p.out) return;
    const uint8_t *const w = p.w + o * p.ldw;
    const float sx = p.xs[0], sw = p.ws[p.w_scales == 1 ? 0 : o], b = p.bias ? load_real(p.bias, p.bias_dtype, o) : 0.f;
    int acc = 0;
    const int vectors = (p.k + 15) / 16;        // (the last one may be part of a vector: its bytes of x are made zeros)
    for (int v0 = lane; v0 < vectors; v0 += 32 * TOKEN_UNROLL) {
        uint4 wv[TOKEN_UNROLL], xv[TOKEN_UNROLL];
#pragma unroll
        for (int u = 0; u < TOKEN_UNROLL; ++u) {
            const int v = v0 + 32 * u;
            wv[u] = xv[u] = make_uint4(0, 0, 0, 0);
            if (v < vectors) {
                asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(wv[u].x), "=r"(wv[u].y), "=r"(wv[u].z), "=r"(wv[u].w)
                             : "l"(w + 16ll * v)
                             : "memory");
                xv[u] = *(const uint4 *)(p.x + 16ll * v);
                if (16 * v + 16 > p.k) xv[u] = first_bytes(xv[u], p.k - 16 * v);
            }
        }
#pragma unroll
        for (int u = 0; u < TOKEN_UNROLL; ++u)
            acc = dot4<SIGNED>(xv[u].w, wv[u].w, dot4<SIGNED>(xv[u].z, wv[u].z, dot4<SIGNED>(xv[u].y, wv[u].y, dot4<SIGNED>(xv[u].x, wv[u].x, acc))));
    }
    acc = __reduce_add_sync(0xffffffffu, acc);
    if (lane == 0) store_real(p.y, p.y_dtype, o, scaled(acc, sx, sw, b));
}

// ----------------------------------------------------------------------------- pairs of blocks, 256 x 256 tiles

struct PairParams {
    ScaledParams s;
    int m_tiles, n_tiles, chunks, stages;
    uint32_t idesc;
    uint64_t desc;
    int align;                     // bytes that every row of y starts at a multiple of, up to 32
    int *status;
    unsigned long long wait_limit;
};

constexpr int PAIR_THREADS = 384;             // producer, issuer, two idle warps, eight that empty the accumulators
constexpr int PAIR_GROUP = 8;                 // tile rows that are walked together: a wave of tiles covers about as many columns
constexpr uint32_t PAIR_STAGE = 2 * 128 * SC_KB;

__device__ __forceinline__ void pair_tile(int t, const PairParams &p, int &m_t, int &n_t) {
    const int per = PAIR_GROUP * p.n_tiles, g = t / per, first = g * PAIR_GROUP, rows = min(PAIR_GROUP, p.m_tiles - first), r = t - g * per;
    n_t = r / rows;
    m_t = first + r - n_t * rows;
}
__device__ __forceinline__ void store_words(void *p, const uint32_t (&w)[8], int bytes) {
    if (bytes == 32) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
        ((uint4 *)p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        ((uint4 *)p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

__global__ void __launch_bounds__(PAIR_THREADS, 1) scaled_pair_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const PairParams p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t *const base = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    ScControl &ctl = *(ScControl *)base;
    float *const factors = (float *)(base + SC_CONTROL);        // two tiles' scales and biases: [2][512]
    const uint32_t ring_at = smem_u32(base + SC_CONTROL + 4096);
    const uint32_t full = smem_u32(&ctl.full[0]), empty = smem_u32(&ctl.empty[0]), tfull = smem_u32(&ctl.tfull[0]), tempty = smem_u32(&ctl.tempty[0]);
    const int warp = uniform((int)(threadIdx.x >> 5)), lane = threadIdx.x & 31;
    const int rank = (int)uniform(cluster_cta_rank()), worker = (int)blockIdx.x >> 1, workers = (int)gridDim.x >> 1;
    const int tiles = p.m_tiles * p.n_tiles, mine = (tiles - worker + workers - 1) / workers;
    const long long uses = (long long)mine * p.chunks;          // of the ring
    const WaitCtx wc = make_wait_ctx(&ctl.abort_flag, p.status, p.wait_limit);
    if (threadIdx.x == 0) {
        ctl.abort_flag = 0;
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(tfull + 8 * a, 1);
            mbar_init(tempty + 8 * a, 16);                      // the eight warps of both blocks
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        prefetch_tensormap(&map_x);
        prefetch_tensormap(&map_w);
    }
    if (warp == 1) tmem_alloc_pair(smem_u32(&ctl.tmem), 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                        // the partner's barriers exist before anything is sent to them
    tc_fence_after();
    const uint32_t tmem = uniform(ctl.tmem);
    grid_dependency_wait();
    grid_launch_dependents();

    if (warp == 0) {
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        long long use = 0;
        for (int t = worker; ok && t < tiles; t += workers) {
            int m_t, n_t;
            pair_tile(t, p, m_t, n_t);
            const int m0 = 256 * m_t + 128 * rank, n0 = 256 * n_t + 128 * rank;
            for (int c = 0; c < p.chunks; ++c, ++use) {
                if (use >= p.stages && !warp_wait(empty + 8 * stage, phase ^ 1, wc, 160)) { ok = false; break; }
                const uint32_t dst = ring_at + (uint32_t)stage * PAIR_STAGE, fb = full + 8 * stage;
                // one barrier for both blocks' copies, in the even block, which announces them all
                if (rank == 0) warp_expect_tx(fb, 2 * PAIR_STAGE);
                tma_load_2d_pair(dst, &map_x, fb, c * SC_KB, m0, lane == 0);
                tma_load_2d_pair(dst + 128 * SC_KB, &map_w, fb, c * SC_KB, n0, lane == 0);
                if (++stage == p.stages) { stage = 0; phase ^= 1; }
            }
        }
        if (!ok) {
            const unsigned long long t0 = clock64();            // copies in flight land before this block's shared memory may go
            while ((unsigned long long)(clock64() - t0) < 4000000ull) {
            }
        }
    } else if (warp == 1 && rank == 0) {
        int stage = 0, local = 0;
        uint32_t phase = 0;
        bool ok = true;
        long long use = 0;
        const uint32_t desc_hi = (uint32_t)(p.desc >> 32);
        for (int t = worker; ok && t < tiles; t += workers, ++local) {
            const int acc = local & 1;
            if (local >= 2 && !warp_wait(tempty + 8 * acc, ((local >> 1) & 1) ^ 1, wc, 161)) { ok = false; break; }
            tc_fence_after();
            for (int c = 0; c < p.chunks; ++c, ++use) {
                if (!warp_wait(full + 8 * stage, phase, wc, 162)) { ok = false; break; }
                tc_fence_after();
                const uint32_t lo = (uint32_t)p.desc | (((ring_at + (uint32_t)stage * PAIR_STAGE) & 0x3ffffu) >> 4);
                mma_i8_sub_pair4(tmem + 256u * acc, lo, lo + ((128 * SC_KB) >> 4), desc_hi, p.idesc, c != 0 ? 1u : 0u);
                if (use + p.stages < uses) mma_commit_pair(empty + 8 * stage);      // (no arrival that nobody waits for)
                if (++stage == p.stages) { stage = 0; phase ^= 1; }
            }
            if (ok) mma_commit_pair(tfull + 8 * acc);
        }
        if (!ok && local > 0) {
            const unsigned long long t0 = clock64();            // the tensor pipe finishes what was issued before its memory goes
            while ((unsigned long long)(clock64() - t0) < 4000000ull) {
            }
        }
    } else if (warp >= 4) {
        const int quad = warp & 3, half = (warp - 4) >> 2, t256 = (int)threadIdx.x - 128;
        const int size = p.s.y_dtype == F8_F32 ? 4 : 2;
        int local = 0;
        // a tile's scales and bias come while the tile before it leaves
        float next_w = 0.f, next_b = 0.f, next_x = 0.f;
        auto prefetch = [&](int t) {
            if (t >= tiles) return;
            int m_t, n_t;
            pair_tile(t, p, m_t, n_t);
            const int o = 256 * n_t + t256, m = 256 * m_t + 128 * rank + 32 * quad + lane;
            next_w = o < p.s.out ? p.s.ws[p.s.w_scales == 1 ? 0 : o] : 0.f;
            next_b = p.s.bias && o < p.s.out ? load_real(p.s.bias, p.s.bias_dtype, o) : 0.f;
            next_x = m < p.s.n ? p.s.xs[p.s.x_scales == 1 ? 0 : m] : 0.f;
        };
        prefetch(worker);
        for (int t = worker; t < tiles; t += workers, ++local) {
            int m_t, n_t;
            pair_tile(t, p, m_t, n_t);
            const int acc = local & 1, n0 = 256 * n_t, m = 256 * m_t + 128 * rank + 32 * quad + lane;
            float *const f = factors + 512 * acc;
            f[t256] = next_w;
            f[256 + t256] = next_b;
            const float sx = next_x;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            prefetch(t + workers);
            if (!warp_wait(tfull + 8 * acc, (local >> 1) & 1, wc, 163)) continue;      // (the others may wait at the barrier above)
            tc_fence_after();
            const uint32_t from = tmem + ((uint32_t)(32 * quad) << 16) + 256u * acc + 128u * half;
            char *const y = (char *)p.s.y + ((long long)m * p.s.ldy + n0 + 128 * half) * size;
#pragma unroll 1
            for (int c = 0; c < 128; c += 16) {
                int v[16];
                tmem_ld16(from + c, v);
                tmem_ld_wait16(v);
                if (c == 112) {                                 // the accumulator is in registers: the next tile but one may have it
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        if (rank == 0) mbar_arrive(tempty + 8 * acc);
                        else mbar_arrive_cluster(tempty + 8 * acc, 0);
                    }
                }
                const int o = n0 + 128 * half + c;
                float r[16];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float4 w4 = *(const float4 *)(f + 128 * half + c + 4 * q), b4 = *(const float4 *)(f + 256 + 128 * half + c + 4 * q);
                    r[4 * q] = scaled(v[4 * q], sx, w4.x, b4.x);
                    r[4 * q + 1] = scaled(v[4 * q + 1], sx, w4.y, b4.y);
                    r[4 * q + 2] = scaled(v[4 * q + 2], sx, w4.z, b4.z);
                    r[4 * q + 3] = scaled(v[4 * q + 3], sx, w4.w, b4.w);
                }
                if (m >= p.s.n) {                               // a lane without a row
                } else if (p.align >= 16 && o + 16 <= p.s.out) {
                    uint32_t w[8];
                    if (size == 4) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
#pragma unroll
                            for (int q = 0; q < 8; ++q) w[q] = __float_as_uint(r[8 * h + q]);
                            store_words(y + (c + 8 * h) * 4, w, p.align);
                        }
                    } else {
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            if (p.s.y_dtype == F8_F16) {
                                const __half2 h2 = __floats2half2_rn(r[2 * q], r[2 * q + 1]);
                                w[q] = *(const uint32_t *)&h2;
                            } else {
                                const __nv_bfloat162 h2 = __floats2bfloat162_rn(r[2 * q], r[2 * q + 1]);
                                w[q] = *(const uint32_t *)&h2;
                            }
                        }
                        store_words(y + c * 2, w, p.align);
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < 16; ++q)
                        if (o + q < p.s.out) store_real(p.s.y, p.s.y_dtype, (long long)m * p.s.ldy + o + q, r[q]);
                }
                __syncwarp();                                   // the next load, and the barrier of the next tile, take all lanes together
            }
        }
    }
    __syncwarp();
    __syncthreads();
    cluster_sync_all();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem, 512);
    }
}

// ----------------------------------------------------------------------------- host side

std::atomic<PFN_cuTensorMapEncodeTiled_v12000> g_encode{nullptr};

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
    PFN_cuTensorMapEncodeTiled_v12000 f = g_encode.load(std::memory_order_acquire);
    if (f) return f;
    void *q = nullptr;
    cudaDriverEntryPointQueryResult qr;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &q, cudaEnableDefault, &qr) != cudaSuccess || !q || qr != cudaDriverEntryPointSuccess) return nullptr;
    f = (PFN_cuTensorMapEncodeTiled_v12000)q;
    g_encode.store(f, std::memory_order_release);
    return f;
}

// rows x k bytes, ld apart, in boxes of 128 bytes by box_rows
bool encode(CUtensorMap *map, const void *p, long long rows, int k, long long ld, int box_rows) {
    PFN_cuTensorMapEncodeTiled_v12000 f = encoder();
    if (!f) return false;
    if (rows == 1) ld = ((long long)k + 15) / 16 * 16;      // (no second row to be elsewhere)
    cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
    cuuint32_t box[2] = {SC_KB, (cuuint32_t)box_rows}, step[2] = {1, 1};
    return f(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int sm_count(int dev) {
    static std::atomic<int> sms[64];
    int v = sms[dev].load(std::memory_order_relaxed);
    if (!v) {
        if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
        sms[dev].store(v, std::memory_order_relaxed);
    }
    return v;
}

// The opt-in to more shared memory than usual is an attribute of each kernel on each device.
template <auto KERNEL>
cudaError_t allow_smem(int dev) {
    static std::atomic<bool> ready[64];
    if (ready[dev].load(std::memory_order_relaxed)) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
    if (e == cudaSuccess) ready[dev].store(true, std::memory_order_relaxed);
    return e;
}

template <typename P>
cudaError_t launch_clusters(void (*kernel)(const CUtensorMap, const CUtensorMap, const P), int grid, int cluster, int threads, size_t smem, cudaStream_t st,
                            const CUtensorMap &mx, const CUtensorMap &mw, const P &p) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, mx, mw, p);
}

// y may be written in words of four elements wherever the column is a multiple of four
bool wide_rows(const ScaledParams &p) {
    const int size = real_size(p.y_dtype);
    return ((uintptr_t)p.y & (uintptr_t)(4 * size - 1)) == 0 && (p.n == 1 || (p.ldy & 3) == 0);
}

template <int BN, bool SOFT>
cudaError_t launch_split(const ScaledParams &s, bool x_signed, int split, int *status, int dev, cudaStream_t st) {
    SplitParams p;
    p.s = s;
    p.m_tiles = (s.n + 127) / 128;
    p.chunks = (s.k + SC_KB - 1) / SC_KB;
    p.split = split;
    p.a_rows = std::min(128, (s.n + 7) / 8 * 8);
    const int tiles = p.m_tiles * ((s.out + BN - 1) / BN), uses = (p.chunks + split - 1) / split;
    p.soft_warps = (p.a_rows + BN + 15) / 16;
    p.slots = p.soft_warps <= 9 ? 8 : 4;
    const size_t raw = SOFT ? ((size_t)p.slots * p.soft_warps * SOFT_RAW + 1023) / 1024 * 1024 : 0;
    const size_t stage = (size_t)(p.a_rows + BN) * SC_KB, head = 3 * 1024 + raw, slack = (size_t)(128 - p.a_rows) * SC_KB;
    const size_t partial = (size_t)std::min(128, s.n) * (BN + 4) * 4;
    // a block to an SM gets a ring of its whole share if that fits; two to an SM get half the memory each
    const size_t room = (!SOFT && tiles * split > sm_count(dev) ? SC_SMEM / 2 - 1024 : SC_SMEM) - head - slack;
    p.stages = std::max(1, std::min({uses, SC_MAX_STAGES, (int)(room / stage)}));
    const size_t smem = 1024 + head + std::max(p.stages * stage + slack, partial);
    p.idesc = (2u << 4) | ((x_signed ? 1u : 0u) << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | (8u << 24);
    p.desc = smem_desc_hi(SC_KB);
    p.wide = wide_rows(s);
    p.status = status;
    p.wait_limit = f8_wait_limit_cycles();
    CUtensorMap mx, mw;
    if (SOFT) {
        memset(&mx, 0, sizeof(mx));
        memset(&mw, 0, sizeof(mw));
    } else if (!encode(&mx, s.x, s.n, s.k, s.ldx, p.a_rows) || !encode(&mw, s.w, s.out, s.k, s.ldw, BN)) {
        return cudaErrorNotSupported;
    }
    const cudaError_t e = allow_smem<scaled_split_kernel<BN, SOFT>>(dev);
    if (e != cudaSuccess) return e;
    return launch_clusters(scaled_split_kernel<BN, SOFT>, tiles * split, split, SPLIT_THREADS + (SOFT ? SOFT_THREADS : 0), smem, st, mx, mw, p);
}

cudaError_t launch_pairs(const ScaledParams &s, bool x_signed, int *status, int dev, cudaStream_t st) {
    PairParams p;
    p.s = s;
    p.m_tiles = (s.n + 255) / 256;
    p.n_tiles = (s.out + 255) / 256;
    p.chunks = (s.k + SC_KB - 1) / SC_KB;
    p.stages = 6;
    p.idesc = (2u << 4) | ((x_signed ? 1u : 0u) << 7) | (1u << 10) | ((256u >> 3) << 17) | ((256u >> 4) << 24);
    p.desc = smem_desc_hi(SC_KB);
    const int size = real_size(s.y_dtype);
    const uintptr_t off = (uintptr_t)s.y | (uintptr_t)(s.n > 1 ? s.ldy * size : 0);
    p.align = (off & 31) == 0 ? 32 : (off & 15) == 0 ? 16 : 1;
    p.status = status;
    p.wait_limit = f8_wait_limit_cycles();
    CUtensorMap mx, mw;
    if (!encode(&mx, s.x, s.n, s.k, s.ldx, 128) || !encode(&mw, s.w, s.out, s.k, s.ldw, 128)) return cudaErrorNotSupported;
    cudaError_t e = allow_smem<scaled_pair_kernel>(dev);
    if (e != cudaSuccess) return e;
    const size_t smem = 1024 + SC_CONTROL + 4096 + (size_t)p.stages * PAIR_STAGE;
    // persistent pairs: no more than the device holds at once
    static std::atomic<int> most[64];
    int pairs = most[dev].load(std::memory_order_relaxed);
    if (!pairs) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(2 * (unsigned)(sm_count(dev) / 2));
        cfg.blockDim = dim3(PAIR_THREADS);
        cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&pairs, scaled_pair_kernel, &cfg);
        if (e != cudaSuccess) return e;
        if (pairs <= 0) return cudaErrorNotSupported;
        most[dev].store(pairs, std::memory_order_relaxed);
    }
    return launch_clusters(scaled_pair_kernel, 2 * std::min(pairs, p.m_tiles * p.n_tiles), 2, PAIR_THREADS, smem, st, mx, mw, p);
}

// Which kernel and tile, by an estimate of the time in microseconds, fitted to calls of 1 to 8192 rows on a B200 (within 15 % of most):
//   split   3.3 for the launch, then the slower of the blocks' chunks (one of BN columns takes 0.12 or 0.15, plus the rows of x it
//           brings; more blocks than SMs share them) and the memory (5.7 or 6.2 TB/s, if enough SMs ask), then the tile's way out, and for a split
//           the exchange.  Eight blocks of a cluster only pay with few rows and no more blocks than SMs.
//   soft    (rows fetched by warps) one block to an SM, 0.55 or 0.72 a chunk and the rows of x
//   pairs   7, then rounds of tiles of 0.29 a chunk, at least 3 for the tile's way out
// Measured (us): 1 x 4096 x 4096 split by 1 / 2 / 4 / 8 at 64 columns 8.3 / 7.2 / 6.7 / 7.7; 256 x 2048 x 1000 7.9 / 6.5 / 5.4 / 7.7; 1 x 8192 x 28672
// 64 columns 42.6, 128 columns 38.7; 512 x 4096 x 4096 split 15.1, pairs 15.5; 1024 x 4096 x 4096 split 21.9, pairs 16.9; soft 1 x 4097 x 4096 at 128
// columns 28.8 / 17.6 / 13.0 / 26.5, 4096 x 4097 x 8192 64 columns 872, 128 columns 529.
struct ScaledCut { int bn, split; };
ScaledCut scaled_cut(const ScaledParams &s, int sms, bool soft) {
    const double chunks = (s.k + SC_KB - 1) / SC_KB, m_tiles = ((long long)s.n + 127) / 128, rows = std::min(128ll, ((long long)s.n + 7) / 8 * 8);
    const double bytes = (double)s.n * s.k + (double)s.out * s.k + (double)s.n * s.out * real_size(s.y_dtype);
    const double pair_tiles = (double)(((long long)s.n + 255) / 256) * (((long long)s.out + 255) / 256);
    ScaledCut best = {256, 1};
    double least = soft ? 1e300 : 7.0 + std::ceil(pair_tiles / (sms / 2)) * std::max(chunks * 0.29, 3.0);
    for (int bn = 64; bn <= 128; bn *= 2) {
        const double tiles = m_tiles * (((long long)s.out + bn - 1) / bn), out = 1.1 * rows * bn / 8192;
        for (int split = 1; split <= 8 && (split == 1 || chunks >= (soft ? 1 : 4) * split); split *= 2) {
            const double share = tiles * split / sms, load = std::max(share, 1.0), uses = std::ceil(chunks / split);
            double t;
            if (soft) {
                t = 0.5 + std::ceil(share) * (3.0 + uses * (bn == 64 ? 0.55 + 0.002 * rows : 0.72 + 0.002 * rows) + out / split);
            } else {
                const double stream = load * uses * (bn == 64 ? 0.115 + 0.0009 * rows : 0.15 + 0.0013 * rows);
                t = 3.3 + std::max(stream, bytes / (bn == 64 ? 5.7e6 : 6.2e6) / std::min(share, 1.0)) + load * out / split;
            }
            if (split > 1) t += 0.4 + rows / 128 * 1.2;
            if (split == 8) t += rows / 128 * 3 + (share > 1 ? 2 : 0);
            if (t < least) {
                least = t;
                best = {bn, split};
            }
        }
    }
    return best;
}

cudaError_t launch_scaled(const ScaledParams &s, bool x_signed, int *status_word, cudaStream_t st) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    const int sms = sm_count(dev);
    if (!status_word || sms <= 0) return cudaErrorMemoryAllocation;
    // blocks of a launch: beyond this neither matrix would fit the device's memory
    if (((long long)s.n + 127) / 128 * (((long long)s.out + 63) / 64) * 8 > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    const bool soft = (((uintptr_t)s.x | (uintptr_t)s.w) & 15) || (s.n > 1 && (s.ldx & 15)) || (s.out > 1 && (s.ldw & 15));
    // One token: a warp a row of w.  Few long rows leave it without enough loads on their way: 16384 x 256 8.5 us, split kernel 6.1.
    if (!soft && s.n == 1 && (s.k <= 4096 || s.out >= 4096)) {
        const dim3 grid((unsigned)(((long long)s.out + TOKEN_THREADS / 32 - 1) / (TOKEN_THREADS / 32)));
        return x_signed ? launch_early(scaled_token_kernel<true>, grid, TOKEN_THREADS, 0, st, s) : launch_early(scaled_token_kernel<false>, grid, TOKEN_THREADS, 0, st, s);
    }
    if (!soft) {
        const ScaledCut cut = scaled_cut(s, sms, false);
        e = cut.bn == 256   ? launch_pairs(s, x_signed, status_word, dev, st)
            : cut.bn == 128 ? launch_split<128, false>(s, x_signed, cut.split, status_word, dev, st)
                            : launch_split<64, false>(s, x_signed, cut.split, status_word, dev, st);
        if (e != cudaErrorNotSupported) return e;       // a matrix no tensor map describes: by the warps
    }
    const ScaledCut cut = scaled_cut(s, sms, true);
    if (cut.bn == 128) return launch_split<128, true>(s, x_signed, cut.split, status_word, dev, st);
    return launch_split<64, true>(s, x_signed, cut.split, status_word, dev, st);
}

}   // namespace

extern "C" f8_status f8_linear_scaled(const f8_scaled_desc *desc, const void *x, const float *x_scale, const int8_t *w, const float *w_scale,
                                      const void *bias, void *y, void *cuda_stream) {
    if (!desc) return f8_set_error(F8_ERR_NULL, "descriptor is NULL");
    f8_scaled_desc d = *desc;
    if (d.n < 0 || d.k <= 0 || d.out <= 0 || d.n > 0x7fffff00 || d.out > 0x7fffff00)
        return f8_set_error(F8_ERR_SHAPE, "n >= 0, k > 0 and out > 0 are needed, n and out at most 2^31 - 256");
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
    const cudaError_t e = launch_scaled(p, d.x_dtype == F8_S8, f8_status_word(), (cudaStream_t)cuda_stream);
    if (e != cudaSuccess) return f8_set_error(F8_ERR_CUDA, cudaGetErrorString(e));
    return F8_OK;
}
