// The linear encoder f(s) = W s and the scores S = Q P^T in 8-bit integers, for a model that has been trained:
//
//     scale_i = max_j |x_ij| (1/127)    q_ij = x_ij / scale_i to the nearest integer, ties to even
//     out_ij  = a_scale_i b_scale_j sum_k A_ik B_jk
//
// gc_quantize_rows is bound by memory: a row is read once (kept in registers), written at a byte per value; 131072 x 768
// bf16 48.4 us, 6.25 TB/s.
// gc_matmul_i8 runs on the tensor cores (tcgen05, kind::i8: exact products and 32-bit integer sums).  Long contractions
// are bound by the products (16384 x 768 x 4096 37 us, 2.8 POP/s; 8192 x 8192 x 4096 163 us, 3.4), short ones by the stores of the
// result (4096 x 8192 x 768 to fp32 31 us, of which 134 MB take 20.5; to bf16 24), few rows of A by reading B (1 x 131072 x 768 18.7 us,
// 5.4 TB/s).  These are times of a call in a graph; called back to back the first is 44 us and the fp32 one 38, since the clock
// falls under the power limit.  Short contractions with bf16 outputs stay farther from their floors (8192 x 768 x 768
// 7.7 us against 3.0, 60000 x 768 x 768 32.4 against 21.8), and so do few tiles of long ones (500 x 500 x 8192 11.4 against
// 1.4: clusters share contractions of up to 64 rows only).
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
constexpr int QZ_BLOCKS = 4;               // to an SM: 3 and 5 are 4 to 20 % slower for nearly all widths
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
            if (BF16) asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(w[e] & 0x7fff7fffu));
            else      m = max(m, w[e] & 0x7fffffffu);
        return m;
    }
};
// The 8-bit integers of a piece: x * inv rounded to integers, r.
// fp32 rows: r is the nearest integer to x / scale if the remainder x - r scale is below half a scale.  The remainder is
// exact (one fused multiply-add: x * inv misses the quotient by less than 2^-15, and the difference has no bits below half of
// scale's last), so where one of the eight is that large, comparing it with scale / 2 decides.
// bf16 rows: see reciprocal().  Rows that neither serves (scales below 2^-100, whose 1 / s may be infinite) form the
// quotients in fp64.
__device__ __noinline__ uint32_t exact_i8(float x, float scale) {
    const double q = rint((double)x / (double)scale);
    return (uint32_t)(int)fmin(fmax(q, -127.0), 127.0);
}
template <bool BF16>
__device__ __forceinline__ uint2 to_i8(const Piece<BF16>& x, float inv, float scale, bool wide) {
    uint32_t m[8];
    float most = 0.f;
    const uint64_t inv2 = pack2(inv, inv), magic2 = pack2(MAGIC, MAGIC), minus2 = pack2(-1.f, -1.f);
    const uint64_t scale2 = pack2(scale, scale);
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const uint64_t v = pack2(x.at(e), x.at(e + 1)), t = fma2(v, inv2, magic2);
        float a, b;
        if (!BF16) {
            unpack2(fma2(fma2(t, minus2, magic2), scale2, v), a, b);
            most = fmaxf(most, fmaxf(fabsf(a), fabsf(b)));
        }
        unpack2(t, a, b);
        m[e] = __float_as_uint(a);
        m[e + 1] = __float_as_uint(b);
    }
    if (wide) {
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = exact_i8(x.at(e), scale);
    } else if (!BF16 && most >= 0.5f * scale) {
        const float half = 0.5f * scale;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float rest = fmaf(MAGIC - __uint_as_float(m[e]), scale, x.at(e)), far = fabsf(rest);
            if (far > half || (far == half && (m[e] & 1u))) m[e] += rest > 0.f ? 1u : 0xffffffffu;
        }
    }
    return make_uint2(__byte_perm(__byte_perm(m[0], m[1], 0x0040), __byte_perm(m[2], m[3], 0x0040), 0x5410),
                      __byte_perm(__byte_perm(m[4], m[5], 0x0040), __byte_perm(m[6], m[7], 0x0040), 0x5410));
}

// inv, 1 / s within 2^-21 of itself; false where the row has to form its quotients in fp64.
// bf16 rows: x = X 2^a and amax = A 2^b with integers X, A below 256, so 127 x / amax lies either halfway between two
// integers or at least 2^-16 of itself away from there, while x / s and x * inv miss it by less than 2^-20.  So x * inv rounds
// as x / s does unless 127 x / amax = h is such a half.  Then x / s = h (amax / 127 s) and x * inv = h (amax inv / 127), and inv is
// moved until both factors are on the same side of 1, or both are 1 (ties to even: one rounding, of the fused
// multiply-add).  Two differences with exact signs for a row replace a remainder for every value, of which nearly
// every piece of a warp has one to look at (131072 x 768: 61 us with that, a warp to a row).
template <bool BF16>
__device__ __forceinline__ bool reciprocal(float s, float amax, float& inv) {
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
    if (!BF16) return true;
    const float eps = fmaf(-127.f, s, amax);
    auto side = [&] { return fmaf(amax, inv, -127.f); };
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float at = side();
        if (eps > 0.f && at <= 0.f) inv = __uint_as_float(__float_as_uint(inv) + 1u);
        if (eps < 0.f && at >= 0.f) inv = __uint_as_float(__float_as_uint(inv) - 1u);
    }
    const float at = side();
    return eps > 0.f ? at > 0.f : eps < 0.f ? at < 0.f : at == 0.f;
}

// LANES lanes (8, 16, a warp or several) to a row; a lane holds KEEP pieces of 8 values of it in registers and reads
// what is beyond them twice.
template <bool BF16, int LANES, int KEEP>
__global__ void __launch_bounds__(QZ_THREADS, QZ_BLOCKS)
quantize_rows_kernel(const void* X, int64_t ldx, int64_t rows, int64_t d, int8_t* q, int64_t ldq, float* scale) {
    constexpr int PER_BLOCK = QZ_THREADS / LANES, STEP = LANES * 8, WARPS = LANES < 32 ? 1 : LANES / 32;
    __shared__ uint32_t warp_max[2][QZ_THREADS / 32];
    const int lane = threadIdx.x % LANES, warp = threadIdx.x >> 5;
    const int64_t k0 = 8 * lane, pitch = ldx * (BF16 ? 2 : 4);
    dep_release();
    dep_wait();
    int turn = 0;
    for (int64_t first = blockIdx.x * (int64_t)PER_BLOCK; first < rows; first += (int64_t)gridDim.x * PER_BLOCK) {
        const int64_t i = first + threadIdx.x / LANES;
        const bool live = i < rows;
        const char* src = static_cast<const char*>(X) + (live ? i : first) * pitch;
        Piece<BF16> x[KEEP];
        uint32_t most = 0;
#pragma unroll
        for (int c = 0; c < KEEP; ++c) x[c].load(src, k0 + c * STEP, d);
#pragma unroll
        for (int c = 0; c < KEEP; ++c) most = x[c].most(most);
        if (LANES == QZ_THREADS) {
            for (int64_t k = k0 + KEEP * STEP; k < d; k += STEP) {
                Piece<BF16> v;
                v.load(src, k, d);
                most = v.most(most);
            }
        }
        if (BF16) most = max(most & 0xffff0000u, most << 16);
        if (LANES < 32) {
#pragma unroll
            for (int o = LANES / 2; o > 0; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
        } else {
            most = __reduce_max_sync(0xffffffffu, most);
        }
        if (WARPS > 1) {                   // (the blocks' rows end together: all threads come here equally often)
            if ((threadIdx.x & 31) == 0) warp_max[turn][warp] = most;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WARPS; ++w) most = max(most, warp_max[turn][warp / WARPS * WARPS + w]);
            turn ^= 1;
        }
        const bool bad = most >= 0x7f800000u;
        const float s = bad ? __uint_as_float(0x7fc00000u) : __uint_as_float(most) * RECIP_127;
        const bool none = bad || s == 0.f;
        float inv = 0.f;
        const bool wide = s < 0x1p-100f || (!none && !reciprocal<BF16>(s, __uint_as_float(most), inv));
        if (!live) continue;
        if (lane == 0) scale[i] = s;
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
        for (int c = 0; c < KEEP; ++c) put(k0 + c * STEP, x[c]);
        if (LANES == QZ_THREADS) {
            for (int64_t k = k0 + KEEP * STEP; k < d; k += STEP) {
                Piece<BF16> v;
                v.load(src, k, d);
                put(k, v);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------------
// Product
// ---------------------------------------------------------------------------------------------------
constexpr int64_t IM_MAX_K = 131071;       // so many products of -128 and -128 fit 31 bits
constexpr int IM_KB = 128;                 // contraction depth of a ring stage: one swizzle row of bytes
constexpr int IM_MAX_ST = 11;
constexpr size_t IM_SMEM = 225 * 1024;
constexpr int IM_EPI = 16;                 // epilogue warps: four to a quarter of the lanes (with two, bf16 outputs stored
                                           // as they are took 38 us at 4096 x 8192 x 768, with four 28)
constexpr int IM_THREADS = 32 * (NPROD + 1 + IM_EPI);
constexpr uint32_t IM_SCALES = 256;        // bytes of a warp: the scales of its 64 columns

// The product as the tensor cores see it: rows of the M side (128 to a CTA) are lanes of tensor memory, rows of the
// N side (bn to a tile) its columns.
//   plain      M: B (channels), N: A (tokens).  32 lanes hold neighbouring outputs and store them as they are.  Few rows
//              of A cost no more than their share of the instruction.
//   staged     bf16 outputs only.  M: A, N: B.  A lane holds neighbouring outputs of a row; blocks of 32 rows x 32
//              columns leave through shared memory with bulk tensor stores: half the words to shared memory that
//              fp32 would take, and no trading of rows between lanes.  (Blocks of 64 columns take twice the buffers,
//              which cost a stage of the ring: 4096 x 8192 x 768 27.2 us against 24.3.)
struct ImParams {
    int64_t rows_m, rows_n;
    int kblocks;
    int bn;                                // rows of the N side in a tile: a multiple of 16 (pairs: of 32; staged: of
                                           // 64) up to 256
    int stages;
    int tiles_m, tiles_n;
    int once;                              // the M side's rows leave the L2 first
    const float* m_scale;
    const float* n_scale;
    void* out;
    int64_t ldo;
    int64_t whole;                         // staged: columns in whole 16 bytes, which is what bulk stores write
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

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// The products of 32 lanes' sums with the scales of the N side's rows (in shared memory) and of the lane's row; the
// order is a_scale first.
template <int G, bool LANE_FIRST>
__device__ __forceinline__ void scale_sums(const uint32_t (&v)[G], uint32_t scales, float lane_scale, float (&f)[G]) {
    const uint64_t mine = pack2(lane_scale, lane_scale);
#pragma unroll
    for (int e = 0; e < G; e += 4) {
        uint64_t s0, s1;
        asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(s0), "=l"(s1) : "r"(scales + 4 * e));
        const uint64_t x = pack2((float)(int)v[e], (float)(int)v[e + 1]);
        const uint64_t y = pack2((float)(int)v[e + 2], (float)(int)v[e + 3]);
        unpack2(LANE_FIRST ? mul2(mul2(x, mine), s0) : mul2(mul2(x, s0), mine), f[e], f[e + 1]);
        unpack2(LANE_FIRST ? mul2(mul2(y, mine), s1) : mul2(mul2(y, s1), mine), f[e + 2], f[e + 3]);
    }
}
// Not staged: one block of G rows of A x this warp's 32 rows of B: v the sums (column e: row of A), `scales` those
// rows' scales.  Stores `n` of the G rows, the first at `row`.
template <int G, bool BF16>
__device__ __forceinline__ void store_block(const uint32_t (&v)[G], uint32_t scales, float sb, const ImParams& p,
                                            int64_t row, int n, int64_t j, int lane) {
    float f[G];
    scale_sums<G, false>(v, scales, sb, f);
    if (BF16) {
        // neighbouring lanes trade a row, so that a lane stores two neighbouring outputs
        const int odd = lane & 1;
        const int64_t jj = j - odd;
        __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(p.out) + (row + odd) * p.ldo + jj;
        const bool both = jj + 1 < p.rows_m;
#pragma unroll
        for (int e = 0; e < G; e += 2) {
            const float got = __shfl_xor_sync(0xffffffffu, odd ? f[e] : f[e + 1], 1);
            const __nv_bfloat162 w = odd ? __floats2bfloat162_rn(got, f[e + 1]) : __floats2bfloat162_rn(f[e], got);
            if (e + odd < n) {
                if (both) *reinterpret_cast<__nv_bfloat162*>(dst) = w;
                else if (jj < p.rows_m) *dst = w.x;
            }
            dst += 2 * p.ldo;
        }
    } else if (j < p.rows_m) {
        float* dst = static_cast<float*>(p.out) + row * p.ldo + j;
        if (n >= G) {
#pragma unroll
            for (int e = 0; e < G; ++e) {
                *dst = f[e];
                dst += p.ldo;
            }
        } else {
#pragma unroll
            for (int e = 0; e < G; ++e) {
                if (e < n) *dst = f[e];
                dst += p.ldo;
            }
        }
    }
}

// Bulk tensor load of rows that leave the L2 first.  (Only for rows that one CTA reads: a load with a policy, be it the
// normal one, of rows that all CTAs read at once took 2500 x 50 x 2000 from 7.5 to 18.3 us.)
__device__ __forceinline__ uint64_t evict_first() {
    uint64_t p;
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
template <bool PAIR>
__device__ __forceinline__ void tma_load_policy(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar,
                                                uint64_t policy) {
    if (PAIR)
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint "
            "[%0], [%1, {%2, %3}], [%4], %5;"
            ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar), "l"(policy) : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint "
            "[%0], [%1, {%2, %3}], [%4], %5;"
            ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar), "l"(policy) : "memory");
}

// PAIR: a cluster of two CTAs owns 256 rows of the M side x bn of the N side, 128 and half of bn loaded by each CTA,
// which holds the accumulators of its 128; otherwise a CTA owns 128 x bn.
template <bool PAIR, bool BF16, bool STAGED>
__global__ void __launch_bounds__(IM_THREADS, 1)
matmul_i8_kernel(const __grid_constant__ CUtensorMap mapM, const __grid_constant__ CUtensorMap mapN,
                 const __grid_constant__ CUtensorMap mapO, const ImParams p) {
    static_assert(BF16 || !STAGED, "fp32 outputs are stored as they are");
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) ImBars bars;
    __shared__ uint32_t tmem_s;
    __shared__ int abort_s;
    volatile int* abort_flag = &abort_s;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    const int rank = PAIR ? (int)cluster_ctarank() : 0;
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int n_rows = PAIR ? p.bn / 2 : p.bn;                 // of the N side that this CTA loads
    const uint32_t stage_bytes = CHUNK_BYTES + (uint32_t)n_rows * 128u;
    if (threadIdx.x == 0) {
        abort_s = 0;
        for (int s = 0; s < IM_MAX_ST; ++s) {
            mbar_init(smem_u32(&bars.full[s]), 1);             // the producer warp whose turn it is (pairs: the leader's)
            mbar_init(smem_u32(&bars.empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&bars.acc_full[b]), 1);
            mbar_init(smem_u32(&bars.acc_free[b]), IM_EPI);
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

    const int64_t total = (int64_t)p.tiles_m * p.tiles_n;
    const int64_t first = PAIR ? blockIdx.x >> 1 : blockIdx.x, by = PAIR ? gridDim.x >> 1 : gridDim.x;
    constexpr int M_ROWS = PAIR ? 256 : 128;
    // the side of fewer tiles runs fastest: its rows stay in the L2 while the other side's pass once
    auto tile_at = [&](int64_t t, int* tm, int* tn) {
        if (p.tiles_n <= p.tiles_m) { *tm = (int)(t / p.tiles_n); *tn = (int)(t - (int64_t)*tm * p.tiles_n); }
        else                        { *tn = (int)(t / p.tiles_m); *tm = (int)(t - (int64_t)*tn * p.tiles_m); }
    };

    if (warp < NPROD) {
        // the two warps take turns with the stages: one alone issues no more than 23 bytes a cycle
        const uint64_t policy = evict_first();
        const uint32_t m_bytes = CHUNK_BYTES, n_bytes = (uint32_t)n_rows * 128u;
        int stage = 0, item = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int64_t t = first; t < total && ok; t += by) {
            int tm, tn;
            tile_at(t, &tm, &tn);
            const int m_row = tm * M_ROWS + rank * 128, n_row = tn * p.bn + rank * n_rows;
            for (int kb = 0; kb < p.kblocks; ++kb, ++item) {
                if ((item & 1) == warp) {
                    ok = mbar_wait(smem_u32(&bars.empty[stage]), phase ^ 1u, abort_flag);
                    if (!ok) break;
                    const uint32_t full = smem_u32(&bars.full[stage]);
                    const uint32_t dst = smem + stage * stage_bytes;
                    const uint32_t full_leader = PAIR ? mapa_u32(full, 0) : full;
                    if (elect_one()) {
                        if (PAIR) {
                            if (rank == 0) mbar_expect_tx(full, 2 * (m_bytes + n_bytes));
                            if (p.once) tma_load_policy<true>(dst, &mapM, kb * IM_KB, m_row, full_leader, policy);
                            else        tma_load_2d_pair(dst, &mapM, kb * IM_KB, m_row, full_leader);
                            tma_load_2d_pair(dst + CHUNK_BYTES, &mapN, kb * IM_KB, n_row, full_leader);
                        } else {
                            mbar_expect_tx(full, m_bytes + n_bytes);
                            if (p.once) tma_load_policy<false>(dst, &mapM, kb * IM_KB, m_row, full, policy);
                            else        tma_load_2d(dst, &mapM, kb * IM_KB, m_row, full);
                            tma_load_2d(dst + CHUNK_BYTES, &mapN, kb * IM_KB, n_row, full);
                        }
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
                    const uint32_t m = desc_lo(smem + stage * stage_bytes, 0);
                    const uint32_t n = desc_lo(smem + stage * stage_bytes + CHUNK_BYTES, 0);
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) mma_i8<PAIR>(acc, m + 2 * k, n + 2 * k, idesc, kb != 0 || k != 0);
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
        // A warp has 32 rows of the M side (a quarter of the lanes) and every fourth block of columns: 64 where they are
        // staged, else 32 (16 in small tiles).
        const int q = warp & 3, ew = warp - (NPROD + 1), group = ew >> 2;
        const int block = STAGED ? 64 : p.bn >= 64 ? 32 : 16;
        const uint32_t after = smem + p.stages * stage_bytes;
        const uint32_t scales = after + (uint32_t)ew * IM_SCALES, buf = after + IM_EPI * IM_SCALES + (uint32_t)ew * 2048u;
        float next_m = 0.f, next_n[2] = {0.f, 0.f};
        // the scales of a tile's rows and of this warp's columns of it, block after block
        auto fetch = [&](int64_t t) {
            if (t >= total) return;
            int tm, tn;
            tile_at(t, &tm, &tn);
            const int64_t i = (int64_t)tm * M_ROWS + rank * 128 + 32 * q + lane, j0 = (int64_t)tn * p.bn;
            const int n = (int)min((int64_t)p.bn, p.rows_n - j0);
            next_m = i < p.rows_m ? p.m_scale[i] : 0.f;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int c = 32 * x + lane, col = (4 * (c / block) + group) * block + c % block;
                next_n[x] = col < n ? p.n_scale[j0 + col] : 0.f;
            }
        };
        fetch(first);
        int use = 0;
        for (int64_t t = first; t < total; t += by, ++use) {
            int tm, tn;
            tile_at(t, &tm, &tn);
            const int64_t row0 = (int64_t)tm * M_ROWS + rank * 128 + 32 * q, i = row0 + lane;   // the lane's row
            const int64_t j0 = (int64_t)tn * p.bn;
            const int n = (int)min((int64_t)p.bn, p.rows_n - j0);
            const float mine = next_m;
            __syncwarp();                          // every lane has read the last tile's
#pragma unroll
            for (int x = 0; x < 2; ++x)
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(scales + 4 * (32 * x + lane)), "f"(next_n[x]) : "memory");
            __syncwarp();
            fetch(t + by);
            if (!mbar_wait(smem_u32(&bars.acc_full[use & 1]), (uint32_t)(use >> 1) & 1u, abort_flag)) break;
            tc_fence_after();
            const uint32_t src = tmem + (use & 1) * 256 + ((uint32_t)(32 * q) << 16);
            // All of the warp's columns are read at once, so that the accumulator is free before anything is stored:
            // the products of the tile after next start under this one's stores.
            uint32_t v[2][32];
            if (block != 16) {
                tmem_ld32(src + (STAGED ? group * 64 : group * 32), v[0]);
                tmem_ld32(src + (STAGED ? group * 64 + 32 : group * 32 + 128), v[1]);
            } else {
                uint32_t w[16];
                tmem_ld16(src + group * 16, w);
#pragma unroll
                for (int e = 0; e < 16; ++e) v[0][e] = w[e];
            }
            tmem_ld_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars.acc_free[use & 1]));
            if (row0 >= p.rows_m) continue;
            if (STAGED) {
                const int c0 = group * 64;
                if (c0 >= n) continue;
#pragma unroll
                for (int y = 0; y < 2; ++y) {                                // 32 columns each
                    const int c = c0 + 32 * y;
                    float f[32];
                    scale_sums<32, true>(v[y], scales + 128 * y, mine, f);
                    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncwarp();
                    if (j0 + c + 32 > p.whole && p.whole < p.rows_n && i < p.rows_m) {
                        // the columns after the last whole 16 bytes
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const int64_t j = j0 + c + e;
                            if (j >= p.whole && j < p.rows_n)
                                static_cast<__nv_bfloat16*>(p.out)[i * p.ldo + j] = __float2bfloat16_rn(f[e]);
                        }
                    }
                    // 16-byte chunk k of row r lies at chunk k ^ (r >> 1 & 3): the map's 64-byte swizzle
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t w[4];
#pragma unroll
                        for (int z = 0; z < 4; ++z) {
                            const __nv_bfloat162 h = __floats2bfloat162_rn(f[8 * k + 2 * z], f[8 * k + 2 * z + 1]);
                            w[z] = *reinterpret_cast<const uint32_t*>(&h);
                        }
                        const uint32_t at = buf + lane * 64 + ((k ^ (lane >> 1 & 3)) << 4);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                                     ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0 && j0 + c < p.whole) tma_store_2d(&mapO, buf, (int)(j0 + c), (int)row0);
                }
            } else if (block == 32) {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int c = (4 * y + group) * 32;
                    if (c < n) store_block<32, BF16>(v[y], scales + 128 * y, mine, p, j0 + c, n - c, i, lane);
                }
            } else if (group * 16 < n) {
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = v[0][e];
                store_block<16, BF16>(w, scales, mine, p, j0 + group * 16, n - group * 16, i, lane);
            }
        }
        if (STAGED) {
            if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
            __syncwarp();
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

// Few rows of A and few tiles: a cluster of CTAs shares a tile of 128 rows of B x bn rows of A.  Each CTA takes a run of
// the contraction blocks, and its sums of columns c .. go to the CTA that owns them (bn / ctas columns each),
// through shared memory; sums of integers have no order.
constexpr int SP_THREADS = 32 * (NPROD + 1 + 8);
constexpr int SP_MAX_CTAS = 8;
constexpr int SP_MAX_BN = 64;
template <bool BF16>
__global__ void __launch_bounds__(SP_THREADS, 1)
matmul_i8_split_kernel(const __grid_constant__ CUtensorMap mapM, const __grid_constant__ CUtensorMap mapN,
                       const ImParams p, const int ctas) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) ImBars bars;
    __shared__ uint32_t tmem_s;
    __shared__ int abort_s;
    volatile int* abort_flag = &abort_s;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    const int rank = (int)cluster_ctarank();
    const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t stage_bytes = CHUNK_BYTES + (uint32_t)p.bn * 128u;
    const uint32_t sums = smem + p.stages * stage_bytes;           // [source CTA][own column][row of B]
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // this CTA has started
    if (threadIdx.x == 0) {
        abort_s = 0;
        for (int s = 0; s < IM_MAX_ST; ++s) {
            mbar_init(smem_u32(&bars.full[s]), 2);
            mbar_init(smem_u32(&bars.empty[s]), 1);
        }
        mbar_init(smem_u32(&bars.acc_full[0]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(&tmem_s)), "r"((uint32_t)SP_MAX_BN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_s;
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");                // and so have those it will send to
    dep_release();
    dep_wait();

    const int tm = (int)(blockIdx.x / (unsigned)ctas);
    const int kb0 = (int)((int64_t)p.kblocks * rank / ctas), kb1 = (int)((int64_t)p.kblocks * (rank + 1) / ctas);
    const int own = p.bn / ctas;                                   // columns of a CTA
    const int64_t row = (int64_t)tm * 128;
    if (warp < NPROD) {
        const bool is_m = warp == 0;
        const uint32_t bytes = is_m ? CHUNK_BYTES : (uint32_t)p.bn * 128u;
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int kb = kb0; kb < kb1 && ok; ++kb) {
            ok = mbar_wait(smem_u32(&bars.empty[stage]), phase ^ 1u, abort_flag);
            if (!ok) break;
            const uint32_t full = smem_u32(&bars.full[stage]);
            if (elect_one()) {
                mbar_expect_tx(full, bytes);
                tma_load_2d(smem + stage * stage_bytes + (is_m ? 0u : CHUNK_BYTES), is_m ? &mapM : &mapN, kb * IM_KB,
                            is_m ? (int)row : 0, full);
            }
            if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
        for (int n = 0; n < p.stages && ok; ++n) {                 // every load and commit is done when the CTA leaves
            ok = mbar_wait(smem_u32(&bars.empty[stage]), phase ^ 1u, abort_flag);
            if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
    } else if (warp == MMA_WARP) {
        const uint32_t idesc = instr_desc_i8(p.bn, 128);
        int stage = 0;
        uint32_t phase = 0;
        for (int kb = kb0; kb < kb1; ++kb) {
            if (!mbar_wait(smem_u32(&bars.full[stage]), phase, abort_flag)) break;
            tc_fence_after();
            const uint32_t m = desc_lo(smem + stage * stage_bytes, 0);
            const uint32_t n = desc_lo(smem + stage * stage_bytes + CHUNK_BYTES, 0);
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < 4; ++k) mma_i8<false>(tmem, m + 2 * k, n + 2 * k, idesc, kb != kb0 || k != 0);
                tc_commit(smem_u32(&bars.empty[stage]));
                if (kb == kb1 - 1) tc_commit(smem_u32(&bars.acc_full[0]));
            }
            if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
    } else {
        // 32 rows of B, every other 16 columns
        const int q = warp & 3, half = (warp - MMA_WARP - 1) >> 2;
        if (mbar_wait(smem_u32(&bars.acc_full[0]), 0, abort_flag)) {
            __syncwarp();
            tc_fence_after();
            for (int c = 16 * half; c < p.bn; c += 32) {
                uint32_t v[16];
                tmem_ld16(tmem + ((uint32_t)(32 * q) << 16) + c, v);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int to = (c + e) / own, col = (c + e) - to * own;
                    asm volatile("st.shared::cluster.b32 [%0], %1;"
                                 ::"r"(mapa_u32(sums + (uint32_t)(((rank * own + col) * 128 + 32 * q + lane) * 4), to)),
                                   "r"(v[e]) : "memory");
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        // let bulk copies still in flight land before the shared memory is released
        uint64_t t0 = global_ns();
        while (global_ns() - t0 < 200000ull) __nanosleep(1000);
        if (threadIdx.x == 0 && p.dev_status) atomicOr(p.dev_status, GC_DEV_WAIT_LIMIT);
        __syncthreads();
    }
    cluster_sync_all();            // everyone's sums have arrived; nobody sends any more
    if (warp == MMA_WARP) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;"
                     ::"r"(tmem), "r"((uint32_t)SP_MAX_BN) : "memory");
    }
    if (warp > MMA_WARP) {
        const int t = threadIdx.x - 32 * (MMA_WARP + 1), r = t & 127;
        const int64_t j = row + r;
        const float sb = j < p.rows_m ? p.m_scale[j] : 0.f;
        for (int col = t >> 7; col < own; col += 2) {
            const int64_t i = (int64_t)rank * own + col;
            if (i >= p.rows_n || j >= p.rows_m) break;
            const float sa = p.n_scale[i];
            int v[SP_MAX_CTAS];
#pragma unroll
            for (int from = 0; from < SP_MAX_CTAS; ++from) {
                v[from] = 0;
                if (from < ctas)
                    asm volatile("ld.shared.b32 %0, [%1];"
                                 : "=r"(v[from]) : "r"(sums + (uint32_t)(((from * own + col) * 128 + r) * 4)));
            }
            int total = 0;
#pragma unroll
            for (int from = 0; from < SP_MAX_CTAS; ++from) total += v[from];
            const float f = (float)total * sa * sb;
            if (BF16) static_cast<__nv_bfloat16*>(p.out)[i * p.ldo + j] = __float2bfloat16_rn(f);
            else      static_cast<float*>(p.out)[i * p.ldo + j] = f;
        }
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

// Checks a matrix; a single row has no pitch, *ld becomes one that the checks of several rows would pass.
int check_matrix(const void* base, int64_t rows, int64_t cols, int64_t* ld, int es) {
    if (!base) return GC_ERR_NULL;
    if (rows <= 0 || cols <= 0) return GC_ERR_SHAPE;
    if (rows > ((int64_t)1 << 30) || cols > ((int64_t)1 << 30)) return GC_ERR_LIMIT;
    if (rows == 1) *ld = (cols + 15) & ~(int64_t)15;
    if (*ld < cols || *ld > ((int64_t)1 << 36)) return GC_ERR_SHAPE;
    if (((uintptr_t)base & 15) || (*ld * es) % 16 != 0) return GC_ERR_ALIGN;
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

// Row-major bf16 output of whole 16 bytes, boxes of 32 rows x 64 bytes, 64-byte swizzle; what lies past the ends is
// not written.
bool make_map_out(CUtensorMap* map, void* base, int64_t rows, int64_t cols, int64_t ld) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
    cuuint32_t box[2] = {32, 32};
    cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) ==
           CUDA_SUCCESS;
}

struct ImPlan { bool pair, staged; int bn; };

// The tile that costs least by a count of cycles: rounds of tiles, each its products or loads, whichever is longer, or
// its stores where they are longer still, and the stores of the last one.  The constants are fitted to 72 shapes with every
// choice forced, one row to 60000 and contractions of 40 to 8192: 2 % behind the best choice on average, 10 % at
// most, in times that repeat within a few per cent, long products under the power limit within 20.  bf16 outputs
// without staging would be 13 % behind (87 % at most), all of them staged 5 (49).
ImPlan make_im_plan(int64_t rows, int64_t cols, int64_t k, bool bf16) {
    ImPlan best{false, false, 16};
    double least = INFINITY;
    const double kblocks = (double)((k + IM_KB - 1) / IM_KB);
    for (int staged = 0; staged < (bf16 && cols >= 8 ? 2 : 1); ++staged) {
        const int64_t m = staged ? rows : cols, n = staged ? cols : rows;
        for (int pair = 0; pair < 2; ++pair)
            // (a staged block of 64 columns must not reach into the next tile)
            for (int step = staged ? 64 : pair ? 32 : 16, bn = step; bn <= 256 && bn < n + step; bn += step) {
                const int64_t tn = (n + bn - 1) / bn, tm = (m + (pair ? 255 : 127)) / (pair ? 256 : 128);
                const int64_t units = sm_count() / (pair ? 2 : 1);
                const double rounds = (double)((tm * tn + units - 1) / units);
                const double products = pair ? 2.0 * bn : 2.0 * bn + 336;
                const double loads = (CHUNK_BYTES + 128.0 * (pair ? bn / 2 : bn)) / 59;
                const double stores = 800 + 128.0 * bn * (bf16 ? 2.0 / (staged ? 53 : 18) : 4.0 / 65);
                const double cost = rounds * std::max(kblocks * std::max(products, loads) + 500, stores) + 1.33 * stores;
                if (cost < least) {
                    least = cost;
                    best = {pair != 0, staged != 0, bn};
                }
            }
    }
    return best;
}

// CTAs to share a tile of few rows of A (1: none do).  The exchange costs as much as a few contraction blocks, more with
// more rows.  Measured, us with 1 / 4 / 8 CTAs: 1 x 768 x 4096 6.5 / 4.8 / 4.1, 1 x 4096 x 4096 6.8 / 5.5 / -, 1 x 1024 x
// 16384 18.6 / 9.4 / 6.3, 1 x 768 x 2048 4.8 / 4.2 / 3.8, 1 x 768 x 1024 3.6 / 3.8 / 3.6, 16 x 768 x 2048 4.6 / 4.1 / 3.7,
// 64 x 768 x 2048 4.8 / 5.9 / 5.3, 64 x 768 x 4096 6.7 / 6.7 / 5.7, 64 x 4096 x 4096 7.0 / 7.2 / -; two never pay.
int split_ctas(int64_t rows, int64_t cols, int64_t k) {
    const int64_t tiles = (cols + 127) / 128, kblocks = (k + IM_KB - 1) / IM_KB;
    if (rows > SP_MAX_BN || kblocks < (rows <= 16 ? 16 : 32)) return 1;
    if (tiles * 8 <= sm_count()) return 8;
    return rows <= 16 && tiles * 4 <= sm_count() ? 4 : 1;
}
int launch_split(const int8_t* A, int64_t lda, const float* a_scale, const int8_t* B, int64_t ldb, const float* b_scale,
                 int64_t rows, int64_t cols, int64_t k, bool bf16, void* out, int64_t ldo, int ctas, int* dev_status,
                 int dev, cudaStream_t st) {
    ImParams p{};
    p.rows_m = cols; p.rows_n = rows;
    p.m_scale = b_scale; p.n_scale = a_scale;
    p.kblocks = (int)((k + IM_KB - 1) / IM_KB);
    p.bn = (int)((rows + 15) / 16 * 16);
    p.tiles_m = (int)((cols + 127) / 128);
    p.stages = std::min(IM_MAX_ST, (int)((IM_SMEM - 1024 - p.bn * 512) / (CHUNK_BYTES + (size_t)p.bn * 128)));
    p.out = out; p.ldo = ldo; p.dev_status = dev_status;
    CUtensorMap mm, mn;
    if (!make_map_i8(&mm, B, cols, k, ldb, 128) || !make_map_i8(&mn, A, rows, k, lda, p.bn)) return GC_ERR_CUDA;
    static bool configured_on[64] = {false};       // the attribute belongs to (kernel, device)
    if (!configured_on[dev]) {
        if (cudaFuncSetAttribute(matmul_i8_split_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 (int)IM_SMEM) != cudaSuccess ||
            cudaFuncSetAttribute(matmul_i8_split_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 (int)IM_SMEM) != cudaSuccess) {
            cudaGetLastError();
            return GC_ERR_CUDA;
        }
        configured_on[dev] = true;
    }
    const cudaError_t e = launch_chained(bf16 ? matmul_i8_split_kernel<true> : matmul_i8_split_kernel<false>,
                                         dim3((unsigned)p.tiles_m * ctas), SP_THREADS, IM_SMEM, ctas, st, mm, mn, p, ctas);
    if (e == cudaSuccess) return GC_OK;
    cudaGetLastError();
    return GC_ERR_CUDA;
}

}  // namespace
}  // namespace gc

using namespace gc;

extern "C" {

int gc_quantize_rows(const void* X, int64_t ldx, int64_t rows, int64_t d, int dtype, int8_t* q, int64_t ldq,
                     float* scale, void* cuda_stream) {
    if (dtype != GC_F32 && dtype != GC_BF16) return GC_ERR_DTYPE;
    int rc = check_matrix(X, rows, d, &ldx, dtype == GC_BF16 ? 2 : 4);
    if (rc || (rc = check_matrix(q, rows, d, &ldq, 1))) return rc;
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
#define GC_QZ(LANES, KEEP)                                                      \
    (dtype == GC_BF16 ? go(quantize_rows_kernel<true, LANES, KEEP>, QZ_THREADS / LANES) \
                      : go(quantize_rows_kernel<false, LANES, KEEP>, QZ_THREADS / LANES))
    // Many bf16 rows: fewer lanes to a row share what a row costs whatever its width (its maximum's exchange, 1 / s, addresses).
    // Measured, us, as fewer rows take them / as many: 131072 x 768 53.5 / 48.5, 100000 x 256 17.6 / 15.6, 32768 x 512 11.9 / 10.4,
    // 8192 x 768 4.2 / 4.1; 4096 x 768 2.9 / 3.6.
    const bool many = dtype == GC_BF16 && rows >= 48 * (int64_t)sm_count();
#define GC_QZ_MANY(LANES, KEEP) go(quantize_rows_kernel<true, LANES, KEEP>, QZ_THREADS / LANES)
    if (many && d > 128 && d <= 256) e = GC_QZ_MANY(8, 4);
    else if (many && d > 256 && d <= 512) e = GC_QZ_MANY(16, 4);
    else if (many && d > 512 && d <= 768) e = GC_QZ_MANY(16, 6);
    else if (d <= 64) e = GC_QZ(8, 1);
    else if (d <= 128) e = GC_QZ(8, 2);
    else if (d <= 256) e = GC_QZ(16, 2);
    else if (d <= 512) e = GC_QZ(32, 2);
    else if (d <= 768) e = GC_QZ(32, 3);
    else if (d <= 1024) e = GC_QZ(32, 4);
    else if (d <= 2048) e = GC_QZ(64, 4);
    else if (d <= 4096) e = GC_QZ(128, 4);
    else e = GC_QZ(256, 4);
#undef GC_QZ
#undef GC_QZ_MANY
    if (e != cudaSuccess) {
        cudaGetLastError();
        return GC_ERR_CUDA;
    }
    return GC_OK;
}

const char* gc_matmul_i8_plan_name(int64_t rows, int64_t cols, int64_t k, int out_dtype) {
    const int64_t most = (int64_t)1 << 30;
    if ((out_dtype != GC_F32 && out_dtype != GC_BF16) || rows <= 0 || cols <= 0 || k <= 0 || rows > most || cols > most ||
        k > IM_MAX_K)
        return "invalid";
    if (split_ctas(rows, cols, k) > 1) return "tcgen05-split";
    const ImPlan pl = make_im_plan(rows, cols, k, out_dtype == GC_BF16);
    if (pl.staged) return pl.pair ? "tcgen05-pairs-staged" : "tcgen05-staged";
    return pl.pair ? "tcgen05-pairs" : "tcgen05";
}

int gc_matmul_i8(const int8_t* A, int64_t lda, const float* a_scale, const int8_t* B, int64_t ldb,
                 const float* b_scale, int64_t rows, int64_t cols, int64_t k, int out_dtype, void* out, int64_t ldo,
                 int* dev_status, void* cuda_stream) {
    if (out_dtype != GC_F32 && out_dtype != GC_BF16) return GC_ERR_DTYPE;
    int rc = check_matrix(A, rows, k, &lda, 1);
    if (rc || (rc = check_matrix(B, cols, k, &ldb, 1)) ||
        (rc = check_matrix(out, rows, cols, &ldo, out_dtype == GC_BF16 ? 2 : 4)))
        return rc;
    if (!a_scale || !b_scale) return GC_ERR_NULL;
    if (k > IM_MAX_K) return GC_ERR_LIMIT;
    int dev;
    if ((rc = check_device(&dev))) return rc;
    const bool bf16 = out_dtype == GC_BF16;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int ctas = split_ctas(rows, cols, k);
    if (ctas > 1) return launch_split(A, lda, a_scale, B, ldb, b_scale, rows, cols, k, bf16, out, ldo, ctas, dev_status, dev, st);
    const ImPlan pl = make_im_plan(rows, cols, k, bf16);
    ImParams p{};
    p.rows_m = pl.staged ? rows : cols;
    p.rows_n = pl.staged ? cols : rows;
    p.m_scale = pl.staged ? a_scale : b_scale;
    p.n_scale = pl.staged ? b_scale : a_scale;
    p.kblocks = (int)((k + IM_KB - 1) / IM_KB);
    p.bn = pl.bn;
    p.tiles_m = (int)((p.rows_m + (pl.pair ? 255 : 127)) / (pl.pair ? 256 : 128));
    p.tiles_n = (int)((p.rows_n + p.bn - 1) / p.bn);
    const int n_rows = pl.pair ? p.bn / 2 : p.bn;
    // Passages that pass once, before few queries, leave the L2 first: a scan of more rows than it holds finds some of them there
    // again the next time.  Measured, us without / with: 1 x 131072 x 768 19.8 / 18.8, 32 x 131072 x 768 22.0 / 20.9,
    // 64 x 50021 x 1000 15.8 / 14.1, 1 x 262144 x 1024 43.7 / 43.4; where more is written 48 x 131072 x 768 23.7 / 24.4,
    // 128 x 131072 x 768 29.6 / 32.1.
    p.once = !pl.staged && p.tiles_n == 1 && rows * cols * (bf16 ? 2 : 4) <= 20000000;
    const size_t room = IM_SMEM - 1024 - IM_EPI * (IM_SCALES + (pl.staged ? 2048 : 0));
    p.stages = std::min(IM_MAX_ST, (int)(room / (CHUNK_BYTES + (size_t)n_rows * 128)));
    p.out = out; p.ldo = ldo; p.dev_status = dev_status;
    p.whole = cols & ~(int64_t)7;
    CUtensorMap mm, mn, mo;
    if (!make_map_i8(&mm, pl.staged ? A : B, p.rows_m, k, pl.staged ? lda : ldb, 128) ||
        !make_map_i8(&mn, pl.staged ? B : A, p.rows_n, k, pl.staged ? ldb : lda, n_rows) ||
        !(pl.staged ? make_map_out(&mo, out, rows, p.whole, ldo) : (mo = mm, true)))
        return GC_ERR_CUDA;
    using Kernel = void (*)(CUtensorMap, CUtensorMap, CUtensorMap, ImParams);
    static const Kernel kernels[6] = {
        matmul_i8_kernel<false, false, false>, matmul_i8_kernel<true, false, false>,
        matmul_i8_kernel<false, true, false>, matmul_i8_kernel<true, true, false>,
        matmul_i8_kernel<false, true, true>, matmul_i8_kernel<true, true, true>};
    static bool configured_on[64] = {false};       // the attribute belongs to (kernel, device)
    if (!configured_on[dev]) {
        for (const Kernel kernel : kernels)
            if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)IM_SMEM) != cudaSuccess) {
                cudaGetLastError();
                return GC_ERR_CUDA;
            }
        configured_on[dev] = true;
    }
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n, units = sm_count() / (pl.pair ? 2 : 1);
    const dim3 grid((unsigned)std::min(total, units) * (pl.pair ? 2u : 1u));
    const cudaError_t e = launch_chained(kernels[2 * bf16 + 2 * pl.staged + pl.pair], grid, IM_THREADS, IM_SMEM,
                                         pl.pair ? 2 : 1, st, mm, mn, mo, p);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return GC_ERR_CUDA;
    }
    return GC_OK;
}

}  // extern "C"
