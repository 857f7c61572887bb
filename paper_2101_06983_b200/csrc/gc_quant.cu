// The linear encoder f(s) = W s and the scores S = Q P^T in 8-bit integers, for a model that has been trained:
//
//     scale_i = max_j |x_ij| (1/127)    q_ij = x_ij / scale_i to the nearest integer, ties to even
//     out_ij  = a_scale_i b_scale_j sum_k A_ik B_jk
//
// gc_quantize_rows is bound by memory: a row is read once (kept in registers), written at a byte per value.
// gc_matmul_i8 runs on the tensor cores (tcgen05, kind::i8: exact products and 32-bit integer sums).  Rows of B
// (channels, passages) are the M = 128 side of the products and rows of A (tokens, queries) the N side: a row of
// B is then a lane of tensor memory, 32 lanes store 32 neighbouring outputs, and few rows of A
// cost no more than their share of the instruction.
#include <cuda_bf16.h>
#include <math.h>

#include <algorithm>

#include "tc_common.cuh"

namespace gc {
namespace {

// ---------------------------------------------------------------------------------------------------
// Rows to 8 bits
// ---------------------------------------------------------------------------------------------------
constexpr int QZ_THREADS = 256;
constexpr float MAGIC = 12582912.f;        // 1.5 * 2^23: adding it rounds to an integer, left in the low bits

constexpr float RECIP_127 = 1.f / 127.f;   // rounded to fp32

// 8 consecutive values of a row as they lie in memory.
template <bool BF16>
struct Piece {
    uint32_t w[BF16 ? 4 : 8];
    __device__ __forceinline__ float at(int e) const {
        if (!BF16) return __uint_as_float(w[BF16 ? 0 : e]);
        return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    }
    // values k .. k + 7 of a row of d: zeros past its end
    __device__ __forceinline__ void load(const char* row, int64_t k, int64_t d) {
        constexpr int N = BF16 ? 1 : 2;
        if (k + 8 <= d) {
#pragma unroll
            for (int h = 0; h < N; ++h) {
                const uint4 v = *reinterpret_cast<const uint4*>(row + (BF16 ? 2 : 4) * k + 16 * h);
                w[4 * h] = v.x; w[4 * h + 1] = v.y; w[4 * h + 2] = v.z; w[4 * h + 3] = v.w;
            }
            return;
        }
if (BF16) {
            const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + k;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t lo = k + 2 * e < d ? p[2 * e] : 0, hi = k + 2 * e + 1 < d ? p[2 * e + 1] : 0;
                w[e] = lo | hi << 16;
            }
        } else {
            const uint32_t* p = reinterpret_cast<const uint32_t*>(row) + k;
#pragma unroll
            for (int e = 0; e < 4 * N; ++e) w[e] = k + e < d ? p[e] : 0;
        }
    }
    // The bits of the largest |x| seen (bf16: of each half word): infinities and NaN lie above every number.
    __device__ __forceinline__ uint32_t most(uint32_t m) const {
#pragma unroll
        for (int e = 0; e < (BF16 ? 4 : 8); ++e)
            m = BF16 ? __vmaxu2(m, w[e] & 0x7fff7fffu) : max(m, w[e] & 0x7fffffffu);
        return m;
    }
};
// The 8-bit integers of a piece.  x * inv misses x / scale by less than 2^-16 (both are at most 127.5, inv is off
// by 2^-24 of itself): where one of the eight is nearer to a border than that, their quotients are formed in
// fp64, where no two quotients of 24-bit numbers on different sides of a border are the same.
template <bool BF16>
__device__ __forceinline__ uint2 to_i8(const Piece<BF16>& x, float inv, float scale, bool wide) {
    uint32_t m[8];
    float off = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float v = x.at(e), t = fmaf(v, inv, MAGIC);
        m[e] = __float_as_uint(t);
        off = fmaxf(off, fabsf(fmaf(v, inv, -(t - MAGIC))));
    }
    if (wide || off > 0.49998f) {
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {
            uint32_t word = x.w[0];                    // (a fixed index: the piece stays in registers)
#pragma unroll
            for (int k = 1; k < (BF16 ? 4 : 8); ++k) if (k == (BF16 ? e >> 1 : e)) word = x.w[k];
            const float v = __uint_as_float(!BF16 ? word : e & 1 ? word & 0xffff0000u : word << 16);
            const double q = rint((double)v / (double)scale);
            const uint32_t r = (uint32_t)(int)fmin(fmax(q, -127.0), 127.0);
#pragma unroll
            for (int k = 0; k < 8; ++k) if (k == e) m[k] = r;
        }
    }
    return make_uint2(__byte_perm(__byte_perm(m[0], m[1], 0x0040), __byte_perm(m[2], m[3], 0x0040), 0x5410),
                      __byte_perm(__byte_perm(m[4], m[5], 0x0040), __byte_perm(m[6], m[7], 0x0040), 0x5410));
}

// WARPS warps to a row; a lane holds KEEP pieces of 8 values of it in registers, the next row's under way
// meanwhile, and reads what is beyond them twice.
template <bool BF16, int WARPS, int KEEP>
__global__ void __launch_bounds__(QZ_THREADS)
quantize_rows_kernel(const void* X, int64_t ldx, int64_t rows, int64_t d, int8_t* q, int64_t ldq, float* scale) {
    constexpr int PER_BLOCK = QZ_THREADS / 32 / WARPS, STEP = 32 * WARPS * 8;
    __shared__ uint32_t warp_max[2][QZ_THREADS / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t k0 = 8 * (lane + 32 * (warp % WARPS)), pitch = ldx * (BF16 ? 2 : 4);
    const int64_t by = (int64_t)gridDim.x * PER_BLOCK;
    dep_release();
    dep_wait();
    int turn = 0;
    int64_t i = blockIdx.x * (int64_t)PER_BLOCK + warp / WARPS;
    Piece<BF16> x[KEEP], next[KEEP];
    auto fetch = [&](int64_t row) {
        const char* src = static_cast<const char*>(X) + row * pitch;
#pragma unroll
        for (int c = 0; c < KEEP; ++c) next[c].load(src, k0 + (int64_t)c * STEP, d);
    };
    if (i < rows) fetch(i);
    for (; i < rows; i += by) {
        const char* src = static_cast<const char*>(X) + i * pitch;
#pragma unroll
        for (int c = 0; c < KEEP; ++c) x[c] = next[c];
        if (i + by < rows) fetch(i + by);
        uint32_t most = 0;
#pragma unroll
        for (int c = 0; c < KEEP; ++c) most = x[c].most(most);
        for (int64_t k = k0 + (int64_t)KEEP * STEP; k < d; k += STEP) {
            Piece<BF16> v;
            v.load(src, k, d);
            most = v.most(most);
        }
        if (BF16) most = max(most & 0xffff0000u, most << 16);
        most = __reduce_max_sync(0xffffffffu, most);
        if (WARPS > 1) {                   // (all rows of a block end together: one row to a block)
            if (lane == 0) warp_max[turn][warp] = most;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WARPS; ++w) most = max(most, warp_max[turn][w]);
            turn ^= 1;
        }
        const bool bad = most >= 0x7f800000u;
        const float s = bad ? __uint_as_float(0x7fc00000u) : __uint_as_float(most) * RECIP_127;
        const bool none = bad || s == 0.f;
        const bool wide = s < 0x1p-100f;   // 1 / s may be infinite, s itself of few bits
        const float inv = none || wide ? 0.f : 1.f / s;
        if (lane == 0 && warp % WARPS == 0) scale[i] = s;
        int8_t* dst = q + i * ldq;
        auto put = [&](int64_t k, const Piece<BF16>& v) {
            if (k >= d) return;
            const uint2 w = none ? make_uint2(0, 0) : to_i8(v, inv, s, wide);
            if (k + 8 <= d) {
                *reinterpret_cast<uint2*>(dst + k) = w;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (k + e < d) dst[k + e] = (int8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
            }
        };
#pragma unroll
        for (int c = 0; c < KEEP; ++c) put(k0 + (int64_t)c * STEP, x[c]);
        for (int64_t k = k0 + (int64_t)KEEP * STEP; k < d; k += STEP) {
            Piece<BF16> v;
            v.load(src, k, d);
            put(k, v);
        }
    }
}

// ---------------------------------------------------------------------------------------------------
// Product
// ---------------------------------------------------------------------------------------------------
constexpr int IM_KB = 128;                 // contraction depth of a ring stage: one swizzle row of bytes
constexpr int IM_MAX_ST = 11;
constexpr size_t IM_SMEM = 225 * 1024;

struct ImParams {
    int64_t rows, cols;                    // of A (tokens), of B (channels)
    int kblocks;
    int bn;                                // rows of A in a tile: a multiple of 16 (pairs: of 32) up to 256
    int stages;
    int tiles_a, tiles_b;
    const float* a_scale;
    const float* b_scale;
    void* out;
    int64_t ldo;
    int* dev_status;
};
struct ImBars {
    uint64_t full[IM_MAX_ST];              // pairs: the leader's counts the bytes of both CTAs
    uint64_t empty[IM_MAX_ST];
    uint64_t acc_full[2];
    uint64_t acc_free[2];                  // this CTA's epilogue warps have read the accumulator
    uint64_t acc_free_peer[2];             // leader: the same, forwarded from the second CTA
};

// Instruction descriptor, kind::i8: signed 8-bit A and B, both K-major, 32-bit integer sums.
__device__ __forceinline__ uint32_t instr_desc_i8(int n, int m) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
template <bool PAIR>
__device__ __forceinline__ void mma_i8(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, bool acc) {
    if (PAIR) {
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
            "setp.ne.b32 p, %5, 0;\n\t"
            "mov.b64 da, {%1, %4};\n\t"
            "mov.b64 db, {%2, %4};\n\t"
            "tcgen05.mma.cta_group::2.kind::i8 [%0], da, db, %3, p;\n\t}"
            ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(DESC_HI), "r"(acc ? 1 : 0)
            : "memory");
    } else {
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
            "setp.ne.b32 p, %5, 0;\n\t"
            "mov.b64 da, {%1, %4};\n\t"
            "mov.b64 db, {%2, %4};\n\t"
            "tcgen05.mma.cta_group::1.kind::i8 [%0], da, db, %3, p;\n\t}"
            ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(DESC_HI), "r"(acc ? 1 : 0)
            : "memory");
    }
}

// One block of G rows of A x this warp's 32 rows of B: v the sums (column e: row of A), sa the scale of row `lane`
// of the block.  Stores `n` of the G rows, the first at `row`.
template <int G, bool BF16>
__device__ __forceinline__ void store_block(const uint32_t (&v)[G], float sa, float sb, const ImParams& p, int64_t row,
                                            int n, int64_t j, int lane) {
    float f[G];
#pragma unroll
    for (int e = 0; e < G; ++e) f[e] = (float)(int)v[e] * __shfl_sync(0xffffffffu, sa, e) * sb;
    if (BF16) {
        // neighbouring lanes trade a row, so that a lane stores two neighbouring outputs
        const int odd = lane & 1;
        const int64_t jj = j - odd;
        __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(p.out) + (row + odd) * p.ldo + jj;
        const bool both = jj + 1 < p.cols;
#pragma unroll
        for (int e = 0; e < G; e += 2) {
            const float got = __shfl_xor_sync(0xffffffffu, odd ? f[e] : f[e + 1], 1);
            const __nv_bfloat162 w = odd ? __floats2bfloat162_rn(got, f[e + 1]) : __floats2bfloat162_rn(f[e], got);
            if (e + odd < n) {
                if (both) *reinterpret_cast<__nv_bfloat162*>(dst) = w;
                else if (jj < p.cols) *dst = w.x;
            }
            dst += 2 * p.ldo;
        }
    } else {
        float* dst = static_cast<float*>(p.out) + row * p.ldo + j;
        if (j < p.cols) {
#pragma unroll
            for (int e = 0; e < G; ++e) {
                if (e < n) *dst = f[e];
                dst += p.ldo;
            }
        }
    }
}

// PAIR: a cluster of two CTAs owns 256 rows of B x bn rows of A, 128 of B and half of A's loaded by each CTA, which
// holds the accumulators of its 128; otherwise a CTA owns 128 x bn.
template <bool PAIR, bool BF16>
__global__ void __launch_bounds__(NTHREADS, 1)
matmul_i8_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB,
                 const ImParams p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) ImBars bars;
    __shared__ uint32_t tmem_s;
    __shared__ int abort_s;
    volatile int* abort_flag = &abort_s;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    const int rank = PAIR ? (int)cluster_ctarank() : 0;
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int a_rows = PAIR ? p.bn / 2 : p.bn;                 // of A that this CTA loads
    const uint32_t stage_bytes = CHUNK_BYTES + (uint32_t)a_rows * 128u;
    if (threadIdx.x == 0) {
        abort_s = 0;
        for (int s = 0; s < IM_MAX_ST; ++s) {
            mbar_init(smem_u32(&bars.full[s]), 2);             // the two producer warps (pairs: the leader's)
            mbar_init(smem_u32(&bars.empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&bars.acc_full[b]), 1);
            mbar_init(smem_u32(&bars.acc_free[b]), NSOFT);
            mbar_init(smem_u32(&bars.acc_free_peer[b]), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MMA_WARP) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                         ::"r"(smem_u32(&tmem_s)), "r"((uint32_t)TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                         ::"r"(smem_u32(&tmem_s)), "r"((uint32_t)TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = tmem_s;
    dep_release();
    dep_wait();

    const int64_t total = (int64_t)p.tiles_a * p.tiles_b;
    const int64_t first = PAIR ? blockIdx.x >> 1 : blockIdx.x, by = PAIR ? gridDim.x >> 1 : gridDim.x;
    constexpr int B_ROWS = PAIR ? 256 : 128;
    // the side of fewer tiles runs fastest: its rows stay in the L2 while the other side's pass once
    auto tile_at = [&](int64_t t, int* ta, int* tb) {
        if (p.tiles_a <= p.tiles_b) { *tb = (int)(t / p.tiles_a); *ta = (int)(t - (int64_t)*tb * p.tiles_a); }
        else                        { *ta = (int)(t / p.tiles_b); *tb = (int)(t - (int64_t)*ta * p.tiles_b); }
    };

    if (warp < NPROD) {
        const bool is_b = warp == 0;       // warp 0: rows of B, warp 1: rows of A
        const uint32_t bytes = is_b ? CHUNK_BYTES : (uint32_t)a_rows * 128u;
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int64_t t = first; t < total && ok; t += by) {
            int ta, tb;
            tile_at(t, &ta, &tb);
            const int row = is_b ? tb * B_ROWS + rank * 128 : ta * p.bn + rank * a_rows;
            for (int kb = 0; kb < p.kblocks; ++kb) {
                ok = mbar_wait(smem_u32(&bars.empty[stage]), phase ^ 1u, abort_flag);
                if (!ok) break;
                const uint32_t full = smem_u32(&bars.full[stage]);
                const uint32_t dst = smem + stage * stage_bytes + (is_b ? 0u : CHUNK_BYTES);
                const uint32_t full_leader = PAIR ? mapa_u32(full, 0) : full;
                if (elect_one()) {
                    if (PAIR) {
                        if (rank == 0) mbar_expect_tx(full, 2 * bytes);
                        tma_load_2d_pair(dst, is_b ? &mapB : &mapA, kb * IM_KB, row, full_leader);
                    } else {
                        mbar_expect_tx(full, bytes);
                        tma_load_2d(dst, is_b ? &mapB : &mapA, kb * IM_KB, row, full);
                    }
                }
                if (++stage == p.stages) { stage = 0; phase ^= 1u; }
            }
        }
        // every stage given back: no load and no commit is under way when the CTA leaves
        for (int n = 0; n < p.stages && ok; ++n) {
            ok = mbar_wait(smem_u32(&bars.empty[stage]), phase ^ 1u, abort_flag);
            if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
    } else if (warp == MMA_WARP) {
        int use = 0;
        bool ok = true;
        if (rank == 0) {
            const uint32_t idesc = instr_desc_i8(p.bn, PAIR ? 256 : 128);
            int stage = 0;
            uint32_t phase = 0;
            for (int64_t t = first; t < total && ok; t += by, ++use) {
                const uint32_t par = ((uint32_t)(use >> 1) & 1u) ^ 1u;
                ok = mbar_wait(smem_u32(&bars.acc_free[use & 1]), par, abort_flag) &&
                     (!PAIR || mbar_wait(smem_u32(&bars.acc_free_peer[use & 1]), par, abort_flag));
                if (!ok) break;
                tc_fence_after();
                const uint32_t acc = tmem + (use & 1) * 256;
                for (int kb = 0; kb < p.kblocks; ++kb) {
                    ok = mbar_wait(smem_u32(&bars.full[stage]), phase, abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t b = desc_lo(smem + stage * stage_bytes, 0);
                    const uint32_t a = desc_lo(smem + stage * stage_bytes + CHUNK_BYTES, 0);
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) mma_i8<PAIR>(acc, b + 2 * k, a + 2 * k, idesc, kb != 0 || k != 0);
                        if (PAIR) {
                            tc_commit_pair(smem_u32(&bars.empty[stage]));
                            if (kb == p.kblocks - 1) tc_commit_pair(smem_u32(&bars.acc_full[use & 1]));
                        } else {
                            tc_commit(smem_u32(&bars.empty[stage]));
                            if (kb == p.kblocks - 1) tc_commit(smem_u32(&bars.acc_full[use & 1]));
                        }
                    }
                    if (++stage == p.stages) { stage = 0; phase ^= 1u; }
                }
            }
        } else {
            // what the leader waits for: every use but the last two
            int uses = 0;
            for (int64_t t = first; t < total; t += by) ++uses;
            for (; use < uses - 2 && ok; ++use) {
                ok = mbar_wait(smem_u32(&bars.acc_free[use & 1]), (uint32_t)(use >> 1) & 1u, abort_flag);
                if (ok && elect_one()) mbar_arrive_cluster(mapa_u32(smem_u32(&bars.acc_free_peer[use & 1]), 0));
            }
        }
    } else {
        // warp: 32 rows of B (a quarter of the lanes), every other block of 32 rows of A (16 in small tiles)
        const int q = warp & 3, half = (warp - (NPROD + 1)) >> 2;
        const int block = p.bn >= 64 ? 32 : 16;
        int use = 0;
        for (int64_t t = first; t < total; t += by, ++use) {
            int ta, tb;
            tile_at(t, &ta, &tb);
            const int64_t j = (int64_t)tb * B_ROWS + rank * 128 + 32 * q + lane;       // this lane's row of B
            const int64_t i0 = (int64_t)ta * p.bn;
            const int n = (int)min((int64_t)p.bn, p.rows - i0);
            const float sb = j < p.cols ? p.b_scale[j] : 0.f;
            float sa[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int c = (2 * x + half) * block + lane;
                sa[x] = c < n ? p.a_scale[i0 + c] : 0.f;
            }
            if (!mbar_wait(smem_u32(&bars.acc_full[use & 1]), (uint32_t)(use >> 1) & 1u, abort_flag)) break;
            tc_fence_after();
            const uint32_t src = tmem + (use & 1) * 256 + ((uint32_t)(32 * q) << 16);
            const int64_t wrow = (int64_t)tb * B_ROWS + rank * 128 + 32 * q;           // the warp's first
            if (wrow < p.cols) {
                if (block == 32) {
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int c = (2 * x + half) * 32;
                        if (c < n) {
                            uint32_t v[32];
                            tmem_ld32(src + c, v);
                            tmem_ld_wait();
                            store_block<32, BF16>(v, sa[x], sb, p, i0 + c, n - c, j, lane);
                        }
                    }
                } else {
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int c = (2 * x + half) * 16;
                        if (c < n) {
                            uint32_t v[16];
                            tmem_ld16(src + c, v);
                            tmem_ld_wait();
                            store_block<16, BF16>(v, sa[x], sb, p, i0 + c, n - c, j, lane);
                        }
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars.acc_free[use & 1]));
        }
    }

    // ------------------------------ teardown ------------------------------------------------------
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        // let bulk copies still in flight land before the shared memory is released
        uint64_t t0 = global_ns();
        while (global_ns() - t0 < 200000ull) __nanosleep(1000);
        if (threadIdx.x == 0 && p.dev_status) atomicOr(p.dev_status, GC_DEV_WAIT_LIMIT);
        __syncthreads();
    }
    if (PAIR) cluster_meet();       // every load, product, commit and arrival between the CTAs has been waited for
    if (warp == MMA_WARP) {
        tc_fence_after();
        if (PAIR)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;"
                         ::"r"(tmem), "r"((uint32_t)TMEM_COLS) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;"
                         ::"r"(tmem), "r"((uint32_t)TMEM_COLS) : "memory");
    }
}

// ---- host ------------------------------------------------------------------------------------------
// Row-major bytes [rows x k], boxes of box_rows x 128 bytes, 128-byte swizzle, zeros past the ends.
bool make_map_i8(CUtensorMap* map, const void* base, int64_t rows, int64_t k, int64_t ld, int box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld};
    cuuint32_t box[2] = {IM_KB, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int check_matrix(const void* base, int64_t rows, int64_t cols, int64_t ld, int es) {
    if (!base) return GC_ERR_NULL;
    if (rows <= 0 || cols <= 0 || ld < cols || ld > ((int64_t)1 << 36)) return GC_ERR_SHAPE;
    if (rows > ((int64_t)1 << 30) || cols > ((int64_t)1 << 30)) return GC_ERR_LIMIT;
    if (((uintptr_t)base & 15) || (ld * es) % 16 != 0) return GC_ERR_ALIGN;
    return GC_OK;
}
int check_device(int* dev) {
    int major = 0;
    if (cudaGetDevice(dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, *dev) != cudaSuccess) {
        cudaGetLastError();
        return GC_ERR_CUDA;
    }
    if (major != 10) return GC_ERR_ARCH;
    return *dev < 0 || *dev >= 64 ? GC_ERR_CUDA : GC_OK;
}

struct ImPlan { bool pair; int bn; };

// The tile that costs least by a count of cycles: rounds of tiles, each its products, its loads (85 bytes a
// cycle) or its stores (20), whichever is longest, and the stores of the last one.
ImPlan make_im_plan(int64_t rows, int64_t cols, int64_t k, int out_dtype) {
    ImPlan best{false, 16};
    double least = INFINITY;
    const double kblocks = (double)((k + IM_KB - 1) / IM_KB);
    const int most = (int)std::min<int64_t>(256, (rows + 15) / 16 * 16);
    for (int pair = 0; pair < 2; ++pair)
        for (int bn = pair ? 32 : 16; bn <= 256; bn += pair ? 32 : 16) {
            if (bn >= most + (pair ? 32 : 16)) break;
            const int64_t ta = (rows + bn - 1) / bn, tb = (cols + (pair ? 255 : 127)) / (pair ? 256 : 128);
            const int64_t units = sm_count() / (pair ? 2 : 1);
            const double rounds = (double)((ta * tb + units - 1) / units);
            const double products = pair ? std::max(2.0 * bn, 190.0) : 4 * (bn / 2.0 + 44);
            const double loads = (CHUNK_BYTES + 128.0 * (pair ? bn / 2 : bn)) / 85;
            const double stores = 128.0 * bn * (out_dtype == GC_BF16 ? 2 : 4) / 20;
            const double cost = rounds * std::max(kblocks * std::max(products, loads), stores) + stores;
            if (cost < least) {
                least = cost;
                best = {pair != 0, bn};
            }
        }
    return best;
}

}  // namespace
}  // namespace gc

using namespace gc;

extern "C" {

int gc_quantize_rows(const void* X, int64_t ldx, int64_t rows, int64_t d, int dtype, int8_t* q, int64_t ldq,
                     float* scale, void* cuda_stream) {
    if (dtype != GC_F32 && dtype != GC_BF16) return GC_ERR_DTYPE;
    int rc = check_matrix(X, rows, d, ldx, dtype == GC_BF16 ? 2 : 4);
    if (rc || (rc = check_matrix(q, rows, d, ldq, 1))) return rc;
    if (!scale) return GC_ERR_NULL;
    int dev;
    if ((rc = check_device(&dev))) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    auto go = [&](auto kernel, int per_block) {
        const int64_t blocks = (rows + per_block - 1) / per_block, most = 8 * (int64_t)sm_count();
        return launch_chained(kernel, dim3((unsigned)std::min(blocks, most)), QZ_THREADS, 0, 1, st, X, ldx, rows, d, q,
                              ldq, scale);
    };
    cudaError_t e;
#define GC_QUANTIZE(BF16)                                                                                   \
    (d <= 256 ? go(quantize_rows_kernel<BF16, 1, 1>, 8) : d <= 512 ? go(quantize_rows_kernel<BF16, 1, 2>, 8) \
     : d <= 768 ? go(quantize_rows_kernel<BF16, 1, 3>, 8) : d <= 1024 ? go(quantize_rows_kernel<BF16, 1, 4>, 8) \
     : d <= 2048 ? go(quantize_rows_kernel<BF16, 8, 1>, 1) : d <= 4096 ? go(quantize_rows_kernel<BF16, 8, 2>, 1) \
                 : go(quantize_rows_kernel<BF16, 8, 4>, 1))
    e = dtype == GC_BF16 ? GC_QUANTIZE(true) : GC_QUANTIZE(false);
#undef GC_QUANTIZE
    if (e != cudaSuccess) {
        cudaGetLastError();
        return GC_ERR_CUDA;
    }
    return GC_OK;
}

int gc_matmul_i8(const int8_t* A, int64_t lda, const float* a_scale, const int8_t* B, int64_t ldb,
                 const float* b_scale, int64_t rows, int64_t cols, int64_t k, int out_dtype, void* out, int64_t ldo,
                 int* dev_status, void* cuda_stream) {
    if (out_dtype != GC_F32 && out_dtype != GC_BF16) return GC_ERR_DTYPE;
    int rc = check_matrix(A, rows, k, lda, 1);
    if (rc || (rc = check_matrix(B, cols, k, ldb, 1)) ||
        (rc = check_matrix(out, rows, cols, ldo, out_dtype == GC_BF16 ? 2 : 4)))
        return rc;
    if (!a_scale || !b_scale) return GC_ERR_NULL;
    if (k > 131071) return GC_ERR_LIMIT;           // 2^14 (k of -128 times -128) must fit 31 bits
    int dev;
    if ((rc = check_device(&dev))) return rc;
    const ImPlan pl = make_im_plan(rows, cols, k, out_dtype);
    ImParams p{};
    p.rows = rows; p.cols = cols;
    p.kblocks = (int)((k + IM_KB - 1) / IM_KB);
    p.bn = pl.bn;
    p.tiles_a = (int)((rows + p.bn - 1) / p.bn);
    p.tiles_b = (int)((cols + (pl.pair ? 255 : 127)) / (pl.pair ? 256 : 128));
    const int a_rows = pl.pair ? p.bn / 2 : p.bn;
    p.stages = std::min(IM_MAX_ST, (int)((IM_SMEM - 1024) / (CHUNK_BYTES + (size_t)a_rows * 128)));
    p.a_scale = a_scale; p.b_scale = b_scale; p.out = out; p.ldo = ldo; p.dev_status = dev_status;
    CUtensorMap ma, mb;
    if (!make_map_i8(&ma, A, rows, k, lda, a_rows) || !make_map_i8(&mb, B, cols, k, ldb, 128)) return GC_ERR_CUDA;
    using Kernel = void (*)(CUtensorMap, CUtensorMap, ImParams);
    static const Kernel kernels[4] = {matmul_i8_kernel<false, false>, matmul_i8_kernel<false, true>,
                                      matmul_i8_kernel<true, false>, matmul_i8_kernel<true, true>};
    static bool configured_on[64] = {false};       // the attribute belongs to (kernel, device)
    if (!configured_on[dev]) {
        for (const Kernel kernel : kernels)
            if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)IM_SMEM) != cudaSuccess) {
                cudaGetLastError();
                return GC_ERR_CUDA;
            }
        configured_on[dev] = true;
    }
    const int64_t total = (int64_t)p.tiles_a * p.tiles_b, units = sm_count() / (pl.pair ? 2 : 1);
    const dim3 grid((unsigned)std::min(total, units) * (pl.pair ? 2u : 1u));
    const cudaError_t e = launch_chained(kernels[2 * pl.pair + (out_dtype == GC_BF16)], grid, NTHREADS, IM_SMEM,
                                         pl.pair ? 2 : 1, static_cast<cudaStream_t>(cuda_stream), ma, mb, p);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return GC_ERR_CUDA;
    }
    return GC_OK;
}

}  // extern "C"
